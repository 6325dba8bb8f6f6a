// Gated feed-forward block: entry points, the forward, and the gradient of the rows (ffn.h has the formulas).
//
// A wavefront keeps 32 rows of X (and of dOut) in registers as the second operand of every product, so that results come out with the
// rows along the lanes: chunk by chunk of 32 hidden values it forms g^T = Wg^T X^T and u^T (dh^T = Wd dOut^T), applies the activation
// where they lie, and adds Wd^T h^T to its result (Wg dg^T + Wu du^T).  The weights, first laid out by a small launch in the
// order in which the instructions read them (as planes, padded with zeros to whole chunks), come through the LDS for the four
// wavefronts of a workgroup in two halves that take turns: while one is multiplied the other is on its way.
// Nothing of the hidden width is written.  Matrix instructions bound it: 6 (10) N d f operations, sixfold for fp32.
// (Few rows: ffn_few.hip.)
#include <math.h>

#include "rgnn_internal.h"
#include "device_utils.h"
#include "ffn.h"

namespace rgnn {

namespace {

// The weights of all chunks as operands.
struct PackArgs { FfnArgs a; int backward; unsigned char* to; };
template <int D, int PL>
__global__ __launch_bounds__(256) void ffn_pack_kernel(PackArgs p) {
    constexpr int S = D / 16;
    const int sections = p.backward ? 5 : 3;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int lane = (int)(id & 63), s = (int)((id >> 6) % S);
    const int64_t q = (id >> 6) / S;
    const int sec = (int)(q % sections);
    const int64_t chunk = q / sections;
    if (chunk >= p.a.chunks) return;
    float v[8];
    switch (section(p.backward, sec)) {
        case kGate: weight_values<D, PL, kGate>(p.a, (int)chunk, s, lane, v); break;
        case kUp: weight_values<D, PL, kUp>(p.a, (int)chunk, s, lane, v); break;
        case kDown: weight_values<D, PL, kDown>(p.a, (int)chunk, s, lane, v); break;
        case kOut: weight_values<D, PL, kOut>(p.a, (int)chunk, s, lane, v); break;
        case kGateBack: weight_values<D, PL, kGateBack>(p.a, (int)chunk, s, lane, v); break;
        default: weight_values<D, PL, kUpBack>(p.a, (int)chunk, s, lane, v);
    }
    bf16x8 f[PL];
    planes8<PL>(v, f);
    unsigned char* const to = p.to + (((chunk * sections + sec) * S + s) * PL) * kFrag + lane * 16;
#pragma unroll
    for (int k = 0; k < PL; ++k) *reinterpret_cast<bf16x8*>(to + k * kFrag) = f[k];
}

// N operands from memory into the LDS, by all wavefronts of the workgroup
template <int N>
__device__ __forceinline__ void fetch(const unsigned char* from, unsigned char* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < (N + kRowWaves - 1) / kRowWaves; ++i) {
        const int k = i * kRowWaves + wave;
        if (N % kRowWaves == 0 || k < N)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + (size_t)k * kFrag + lane * 16),
                                             (__attribute__((address_space(3))) void*)(lds + k * kFrag), 16, 0, 0);
    }
}
// what this wavefront has under way has arrived, then all have
__device__ __forceinline__ void arrived() {
    __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0)
    __syncthreads();
}

// What a chunk's weights take in the LDS.  One plane: twice, so that one barrier per chunk is enough; three planes (up to 120 KB, and six
// times the instructions to wait behind): once, the halves of a chunk refilled in turn.
template <int D, int PL, bool BWD> struct Weights {
    static constexpr int ops = D / 16 * PL, first = (BWD ? 3 : 2) * ops, second = (BWD ? 2 : 1) * ops;
    static constexpr bool twice = PL == 1;
    static constexpr size_t lds = (size_t)(first + second) * kFrag * (twice ? 2 : 1);
};

// Wavefronts that share a SIMD, and whether the products of chunk c + 1 are issued between the activations of chunk c (the matrix unit and
// the vector unit then work at the same time within a wavefront, which takes the registers of a second set of hidden values).
template <int D, int PL, bool BWD> struct RowsCut {
    static constexpr int per_simd = D == 128 && PL == 3 && BWD ? 1 : 2;
    static constexpr bool ahead = !((BWD && (D == 128 || PL == 3)) || (D == 128 && PL == 3));
    static constexpr int depth = PL == 1 ? (BWD ? 3 : 4) : 2;     // steps of the second products that an operand is read ahead, and one
};

template <int D, int PL, int ACT, bool BWD>
__global__ __launch_bounds__(64 * kRowWaves, (RowsCut<D, PL, BWD>::per_simd)) void ffn_rows_kernel(RowsArgs r) {
    using W = Weights<D, PL, BWD>;
    using Cut = RowsCut<D, PL, BWD>;
    constexpr int S = D / 16, TILES = D / 32;
    using T = typename std::conditional<PL == 1, bf16_t, float>::type;
    extern __shared__ unsigned char lds[];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 31, kh = lane >> 5;
    const int64_t row = ((int64_t)blockIdx.x * kRowWaves + wave) * 32 + m;
    const int c1 = r.a.chunks;
    auto first = [&](int c) { return lds + (W::twice ? (c & 1) * (W::first + W::second) * kFrag : 0); };
    auto second = [&](int c) { return first(c) + W::first * kFrag; };
    auto fetch_first = [&](int c) { if (c < c1) fetch<W::first>(r.packed + (size_t)c * (W::first + W::second) * kFrag, first(c)); };
    auto fetch_second = [&](int c) { if (c < c1) fetch<W::second>(r.packed + ((size_t)c * (W::first + W::second) + W::first) * kFrag, second(c)); };
    fetch_first(0);
    if (W::twice) {
        if (Cut::ahead) fetch_first(1);
        fetch_second(0);
    }
    bf16x8 x[S][PL], dy[BWD ? S : 1][PL];
    v16f y[TILES];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        load_planes8<D, PL>(static_cast<const T*>(r.a.X), row, r.a.rows, 16 * s + 8 * kh, x[s]);
        if constexpr (BWD) load_planes8<D, PL>(static_cast<const T*>(r.a.dOut), row, r.a.rows, 16 * s + 8 * kh, dy[s]);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) clear(y[t]);

    // Operands are read from the LDS a step before they are multiplied.  The compiler would move the reads to their use and wait there; the
    // backward, whose registers are full, is left to it (2M rows, d 128, f 512, bf16, forward: 935 us without the fences, 913 with;
    // 200017 rows, f 341, backward: 119 and 134).
    auto fence = [] { if constexpr (!BWD) __builtin_amdgcn_sched_barrier(0); };
    struct FirstOps { bf16x8 f[BWD ? 3 : 2][PL]; };
    struct SecondOps { bf16x8 f[BWD ? 2 : 1][PL]; };
    auto read_first = [&](const unsigned char* w, int s) {
        FirstOps o;
#pragma unroll
        for (int k = 0; k < (BWD ? 3 : 2); ++k) operand(w + (k * S + s) * PL * kFrag, o.f[k]);
        return o;
    };
    auto read_second = [&](const unsigned char* w, int q) {           // q = TILES s + t
        SecondOps o;
#pragma unroll
        for (int k = 0; k < (BWD ? 2 : 1); ++k) operand(w + (k * S + 2 * (q % TILES) + q / TILES) * PL * kFrag, o.f[k]);
        return o;
    };
    // the s-th sixteen columns' share of the chunk's hidden values
    auto form = [&](const FirstOps& o, int s, Hidden<BWD>& h) {
        mul_add<PL>(o.f[0], x[s], h.g);
        mul_add<PL>(o.f[1], x[s], h.u);
        if constexpr (BWD) mul_add<PL>(o.f[2], dy[s], h.dh);
    };
    // early: the operands of the first steps are on their way already
    constexpr int DEPTH = Cut::depth < S ? Cut::depth : S;
    auto result = [&](int c, SecondOps (&o)[DEPTH], const float (&v)[16], const float (&v2)[16]) {
        bf16x8 p[2][PL], p2[2][PL];
        auto round = [&](int s) {
            planes8<PL>(*reinterpret_cast<const float(*)[8]>(v + 8 * s), p[s]);
            if constexpr (BWD) planes8<PL>(*reinterpret_cast<const float(*)[8]>(v2 + 8 * s), p2[s]);
        };
        round(0);
#pragma unroll
        for (int q = 0; q < S; ++q) {
            if (q + DEPTH - 1 < S) o[(q + DEPTH - 1) % DEPTH] = read_second(second(c), q + DEPTH - 1);
            fence();
            const int s = q / TILES, t = q % TILES;
            mul_add<PL>(o[q % DEPTH].f[0], p[s], y[t]);
            if constexpr (BWD) mul_add<PL>(o[q % DEPTH].f[1], p2[s], y[t]);
            if (q == 0) round(1);
            fence();
        }
    };
    auto read_early = [&](int c, SecondOps (&o)[DEPTH]) {
#pragma unroll
        for (int q = 0; q < DEPTH - 1; ++q) o[q] = read_second(second(c), q);
    };
    auto none = [&](Hidden<BWD>& h) {
        clear(h.g);
        clear(h.u);
        if constexpr (BWD) clear(h.dh);
    };
    // Chunk c from its hidden values: activations, and its share of the result; between the activations chunk c + 1's products (more).
    auto chunk = [&](auto more, int c, Hidden<BWD>& now, Hidden<BWD>& next) {
        arrived();
        if (W::twice) {
            fetch_first(c + 2);
            fetch_second(c + 1);
        } else {
            fetch_second(c);
        }
        float v[16], v2[16];
        SecondOps early[DEPTH];
        if constexpr (more()) {
            none(next);
            FirstOps o = read_first(first(c + 1), 0);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                FirstOps ahead;
                if (s + 1 < S) ahead = read_first(first(c + 1), s + 1);
                if (W::twice && s == S - 1) read_early(c, early);
                fence();
                form(o, s, next);
#pragma unroll
                for (int j = 16 / S * s; j < 16 / S * (s + 1); ++j) {
                    activate<ACT>(now, j, v[j], v2[j]);
                    asm volatile("" : "+v"(v[j]));         // (here, and not together with the others as vectors)
                    if constexpr (BWD) asm volatile("" : "+v"(v2[j]));
                }
                fence();
                o = ahead;
            }
        } else {
            if (W::twice) read_early(c, early);
#pragma unroll
            for (int j = 0; j < 16; ++j) activate<ACT>(now, j, v[j], v2[j]);
        }
        if (!W::twice) {
            arrived();
            fetch_first(c + 2);
            read_early(c, early);
        }
        result(c, early, v, v2);
    };
    Hidden<BWD> a, b;
    if constexpr (Cut::ahead) {
        none(a);
        arrived();
#pragma unroll
        for (int s = 0; s < S; ++s) form(read_first(first(0), s), s, a);
        if (!W::twice) {
            __syncthreads();
            fetch_first(1);
        }
        // (two at a time: the sets of hidden values change places without being moved)
        constexpr std::true_type more;
        constexpr std::false_type last;
        int c = 0;
        for (; c + 2 < c1; c += 2) {
            chunk(more, c, a, b);
            chunk(more, c + 1, b, a);
        }
        if (c + 1 < c1) {
            chunk(more, c, a, b);
            chunk(last, c + 1, b, a);
        } else {
            chunk(last, c, a, b);
        }
    } else {
        for (int c = 0; c < c1; ++c) {
            arrived();
            if (W::twice) {
                fetch_first(c + 1);
                fetch_second(c + 1);
            } else {
                fetch_second(c);
            }
            none(a);
            FirstOps o = read_first(first(c), 0);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                FirstOps ahead;
                if (s + 1 < S) ahead = read_first(first(c), s + 1);
                fence();
                form(o, s, a);
                fence();
                o = ahead;
            }
            if (!W::twice) {
                arrived();
                fetch_first(c + 1);
            }
            float v[16], v2[16];
            SecondOps early[DEPTH];
            read_early(c, early);
#pragma unroll
            for (int j = 0; j < 16; ++j) activate<ACT>(a, j, v[j], v2[j]);
            result(c, early, v, v2);
        }
    }
    store_result<D, PL>(r, 0, row, kh, y);
}

int chunks_of(const rgnn_ffn_desc_t* d) { return (d->hidden + kHid - 1) / kHid; }
constexpr int kBlockRows = 32 * kRowWaves;
size_t packed_bytes(const rgnn_ffn_desc_t* d, bool backward) {
    return align_up((size_t)chunks_of(d) * (backward ? 5 : 3) * (d->width / 16) * (d->dtype == RGNN_BF16 ? 1 : 3) * kFrag);
}
size_t grad_bytes(const rgnn_ffn_desc_t* d) {
    return align_up(sizeof(float) * (size_t)ffn_grad_splits(d) * 3 * d->width * chunks_of(d) * kHid);
}

size_t workspace_bytes(const rgnn_ffn_desc_t* d, bool backward) {
    if (ffn_few(d, backward)) return ffn_few_bytes(d, backward);
    return backward ? std::max(packed_bytes(d, true), grad_bytes(d)) : packed_bytes(d, false);
}

template <int D, int PL, int ACT, bool BWD>
rgnn_status_t launch_rows(const RowsArgs& r, hipStream_t st) {
    constexpr size_t lds = Weights<D, PL, BWD>::lds;
    auto* const kernel = ffn_rows_kernel<D, PL, ACT, BWD>;
    RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds));
    KernelTimer timer(st, BWD ? "ffn_bwd_rows" : "ffn_fwd");
    kernel<<<(unsigned)((r.a.rows + kBlockRows - 1) / kBlockRows), 64 * kRowWaves, lds, st>>>(r);
    RGNN_CHECK_LAUNCH();
    return RGNN_OK;
}

template <bool BWD>
rgnn_status_t rows_pass(const rgnn_ffn_desc_t* d, const FfnArgs& a, void* out, int accumulate, void* workspace, hipStream_t st) {
    unsigned char* const packed = static_cast<unsigned char*>(workspace);
    const RowsArgs r{a, packed, out, nullptr, 1, accumulate};
    auto run = [&]() -> rgnn_status_t {
        RGNN_DISPATCH_FFN(d, {
            {
                const PackArgs p{a, BWD, packed};
                const int64_t threads = (int64_t)a.chunks * (BWD ? 5 : 3) * (D / 16) * 64;
                KernelTimer timer(st, "ffn_pack");
                ffn_pack_kernel<D, PL><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(p);
                RGNN_CHECK_LAUNCH();
            }
            return launch_rows<D, PL, ACT, BWD>(r, st);
        });
    };
    return run();
}

rgnn_status_t check_desc(const rgnn_ffn_desc_t* d) {
    if (!d) RGNN_FAIL(RGNN_EINVAL, "desc is NULL");
    RGNN_TRY(check_rows(d->rows));
    RGNN_TRY(check_dtype(d->dtype));
    
    if (d->width != 32 && d->width != 64 && d->width != 128) RGNN_FAIL(RGNN_EUNSUPPORTED, "width %d not supported (32/64/128)", d->width);
    if (d->hidden < 1) RGNN_FAIL(RGNN_EINVAL, "hidden %d is not positive", d->hidden);
    if (d->hidden > 16384) RGNN_FAIL(RGNN_EUNSUPPORTED, "hidden %d not supported (up to 16384)", d->hidden);
    if (d->activation != RGNN_ACT_RELU && d->activation != RGNN_ACT_SILU) RGNN_FAIL(RGNN_EINVAL, "unknown activation %d", d->activation);
    if (d->flags & ~RGNN_FLAG_ACCUMULATE) RGNN_FAIL(RGNN_EINVAL, "flags: only RGNN_FLAG_ACCUMULATE applies");
    return RGNN_OK;
}

// No written tensor shares memory with another one; all are aligned.
rgnn_status_t check_tensors(std::initializer_list<Span> read, std::initializer_list<Span> written) {
    for (const Span& s : read) RGNN_TRY(check_aligned(s));
    for (const Span* w = written.begin(); w != written.end(); ++w) {
        RGNN_TRY(check_aligned(*w));
        for (const Span& s : read)
            if (w->overlaps(s)) RGNN_FAIL(RGNN_EINVAL, "an output or the workspace overlaps an input");
        for (const Span* v = written.begin(); v != w; ++v)
            if (w->overlaps(*v)) RGNN_FAIL(RGNN_EINVAL, "two outputs, or one and the workspace, overlap");
    }
    return RGNN_OK;
}

}  // namespace

}  // namespace rgnn

using namespace rgnn;

extern "C" rgnn_status_t rgnn_ffn_workspace_bytes(const rgnn_ffn_desc_t* desc, size_t* fwd_workspace, size_t* bwd_workspace) {
    RGNN_TRY(check_desc(desc));
    if (fwd_workspace) *fwd_workspace = workspace_bytes(desc, false);
    if (bwd_workspace) *bwd_workspace = workspace_bytes(desc, true);
    return RGNN_OK;
}

extern "C" rgnn_status_t rgnn_ffn_fwd(const rgnn_ffn_desc_t* desc, const void* X, const void* Wg, const void* Wu, const void* Wd, void* out,
                                      void* workspace, void* stream) {
    RGNN_TRY(check_desc(desc));
    if (desc->rows == 0) return RGNN_OK;
    if (!X || !Wg || !Wu || !Wd || !out) RGNN_FAIL(RGNN_EINVAL, "X, a weight or out is NULL");
    if (!workspace) RGNN_FAIL(RGNN_EWORKSPACE, "workspace is NULL");
    const size_t n = (size_t)desc->rows * desc->width, w = (size_t)desc->hidden * desc->width;
    const int32_t t = desc->dtype;
    RGNN_TRY(check_tensors({span(X, n, t), span(Wg, w, t), span(Wu, w, t), span(Wd, w, t)},
                           {span(out, n, t), Span{static_cast<char*>(workspace), workspace_bytes(desc, false)}}));
    const FfnArgs a{desc->rows, desc->hidden, chunks_of(desc), X, Wg, Wu, Wd, nullptr};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return ffn_few(desc, false) ? ffn_few_fwd(desc, a, out, workspace, st) : rows_pass<false>(desc, a, out, 0, workspace, st);
}

extern "C" rgnn_status_t rgnn_ffn_bwd(const rgnn_ffn_desc_t* desc, const void* X, const void* Wg, const void* Wu, const void* Wd, const void* dOut,
                                      void* dX, void* dWg, void* dWu, void* dWd, void* workspace, void* stream) {
    RGNN_TRY(check_desc(desc));
    const bool grads = dWg || dWu || dWd;
    if (grads && !(dWg && dWu && dWd)) RGNN_FAIL(RGNN_EINVAL, "dWg, dWu and dWd are given together or not at all");
    if (!Wg || !Wu || !Wd) RGNN_FAIL(RGNN_EINVAL, "a weight is NULL");
    if (desc->rows > 0 && (!X || !dOut)) RGNN_FAIL(RGNN_EINVAL, "X or dOut is NULL");
    if (!workspace) RGNN_FAIL(RGNN_EWORKSPACE, "workspace is NULL");
    const size_t n = (size_t)desc->rows * desc->width, w = (size_t)desc->hidden * desc->width;
    const int32_t t = desc->dtype;
    RGNN_TRY(check_tensors({span(X, n, t), span(Wg, w, t), span(Wu, w, t), span(Wd, w, t), span(dOut, n, t)},
                           {span(dX, n, t), span(dWg, w, t), span(dWu, w, t), span(dWd, w, t), Span{static_cast<char*>(workspace), workspace_bytes(desc, true)}}));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const FfnArgs a{desc->rows, desc->hidden, chunks_of(desc), X, Wg, Wu, Wd, dOut};
    const int accumulate = (desc->flags & RGNN_FLAG_ACCUMULATE) != 0;
    if (desc->rows > 0 && ffn_few(desc, true)) return ffn_few_bwd(desc, a, dX, dWg, dWu, dWd, workspace, st);
    if (dX && desc->rows > 0) RGNN_TRY(rows_pass<true>(desc, a, dX, accumulate, workspace, st));
    if (grads && (desc->rows > 0 || !accumulate)) RGNN_TRY(ffn_grad(desc, a, static_cast<float*>(workspace), dWg, dWu, dWd, st));
    return RGNN_OK;
}
