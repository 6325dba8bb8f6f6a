// Gated feed-forward block: entry points and launches (ffn.h has the formulas, ffn_rows.h and ffn_grad.h a workgroup's work, ffn_few.hip the same for
// few rows).
//
// The pass of the rows: a wavefront keeps 32 rows of X (and of dOut) in registers as the second operand of every product, so that results come out with
// the rows along the lanes: chunk by chunk of 32 hidden values it forms g^T = Wg^T X^T and u^T (dh^T = Wd dOut^T), applies the activation
// where they lie, and adds Wd^T h^T to its result (Wg dg^T + Wu du^T).  The weights, first laid out by a small launch in the
// order in which the instructions read them (as planes, padded with zeros to whole chunks), come through the LDS for the four
// wavefronts of a workgroup: bf16 in two places that take turns, fp32 in one whose two halves do.  Nothing of the hidden width is written.
//
// Matrix instructions bound it, 6 N d f operations forward and 16 N d f backward (22 as the hidden values are formed twice), sixfold for fp32; bf16's second
// plane of h, dg and du makes 8 of the 6 and 32 of the 22.  In bf16 up to width 64 the vector instructions are as long, an exponential and a reciprocal per
// hidden value.  Against 1160 TFLOP/s of a large bf16 product, in brackets what the matrix instructions do:
//   forward   2M rows, d 128, f 512, bf16: 1007 us, 781 TFLOP/s (1040); 1M rows, d 64, f 256, bf16: 174 us, 565 (753); fp32: 520 us, 189 (1134)
//   backward  200017 rows, d 128, f 341, bf16: 311 us, 449 (900); 1M rows, d 64, f 256, bf16: 669 us, 392 (783); fp32: 1901 us, 138 (1138)
// From rows held in 8 bits, whose values are one bfloat16 plane, six of the eleven products of fp32 take three plane products instead of six, 48 of 66 in all: 1M rows, d 64, f 256, 1391 us for
// 1805, f 170 1041 for 1368; 300000 rows, d 128, f 341, 1480 for 1820.  In bf16 there is nothing to save, and the weights' gradients unpack a unit of rows once for each
// workgroup of hidden values, a quarter more vector instructions: 200017 rows, d 128, f 341, 320 us for 300.
#include <math.h>

#include "rgnn_internal.h"
#include "device_utils.h"
#include "ffn_grad.h"
#include "ffn_rows.h"

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

template <int D, int PL, int ACT, int GROUPS>
__global__ __launch_bounds__(64 * kRowWaves, (RowsCut<D, PL, false>::per_simd)) void ffn_fwd_kernel(RowsArgs r) {
    extern __shared__ unsigned char lds[];
    rows_block<D, PL, ACT, false, GROUPS>(r, blockIdx.x, lds);
}

// The backward's two passes in one launch: workgroups [0, row_blocks) take the rows, the others the weights' gradients.  Neither waits for
// the other's last workgroups (either by itself, in sum / both in one: 14000 rows, d 64, f 256, bf16, 37.3 / 26.6 us; 200017 rows, d 128, f 341, 322 / 300;
// 1M rows, d 64, f 256, 605 / 592; fp32, 1832 / 1858).
template <int D, int PL, int ACT, bool HELD>
__global__ __launch_bounds__(64 * kRowWaves, (RowsCut<D, PL, true>::per_simd)) void ffn_bwd_kernel(RowsArgs r, FfnGradArgs k, int row_blocks) {
    extern __shared__ unsigned char lds[];
    const int b = (int)blockIdx.x - row_blocks;
    if (b < 0) rows_block<D, PL, ACT, true, 1, HELD>(r, blockIdx.x, lds);
    else grad_block<D, PL, ACT, false, HELD>(k, b % k.splits, b / k.splits, lds);
}

template <typename T>
__global__ __launch_bounds__(256) void ffn_grad_reduce_kernel(FfnGradArgs k, int D) {
    __shared__ float lds[16][64];
    grad_reduce_block<T>(k, D, blockIdx.x, lds);
}

constexpr int64_t kMostRows = 2000000000;      // HIP counts a launch's lanes, two per row, in 32 bits
size_t packed_bytes(const rgnn_ffn_desc_t* d, bool backward) {
    return align_up((size_t)ffn_chunks(d) * (backward ? 5 : 3) * (d->width / 16) * (d->dtype == RGNN_BF16 ? 1 : 3) * kFrag);
}
int grad_splits(const rgnn_ffn_desc_t* d) { return ffn_grad_shares(d, std::max(4, 512 / ffn_grad_groups(d))); }
size_t workspace_bytes(const rgnn_ffn_desc_t* d, bool backward) {
    if (ffn_few(d, backward)) return ffn_few_bytes(d, backward);
    return packed_bytes(d, backward) + (backward ? align_up(sizeof(float) * (size_t)grad_splits(d) * 3 * d->width * ffn_chunks(d) * kHid) : 0);
}

template <int D, int PL>
rgnn_status_t launch_pack(const FfnArgs& a, bool backward, unsigned char* to, hipStream_t st) {
    const int64_t threads = (int64_t)a.chunks * (backward ? 5 : 3) * (D / 16) * 64;
    KernelTimer timer(st, "ffn_pack");
    ffn_pack_kernel<D, PL><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(PackArgs{a, backward, to});
    RGNN_CHECK_LAUNCH();
    return RGNN_OK;
}

rgnn_status_t forward(const rgnn_ffn_desc_t* d, const FfnArgs& a, void* out, void* workspace, hipStream_t st) {
    unsigned char* const packed = static_cast<unsigned char*>(workspace);
    const RowsArgs r{a, packed, out, nullptr, 1, 0};
    RGNN_DISPATCH_FFN(d, {
        RGNN_TRY((launch_pack<D, PL>(a, false, packed, st)));
        auto launch = [&](auto groups) -> rgnn_status_t {
            constexpr size_t lds = Weights<D, PL, false>::lds * groups();
            auto* const kernel = ffn_fwd_kernel<D, PL, ACT, groups()>;
            RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds));
            KernelTimer timer(st, "ffn_fwd");
            kernel<<<(unsigned)((d->rows * groups() + kBlockRows - 1) / kBlockRows), 64 * kRowWaves, lds, st>>>(r);
            RGNN_CHECK_LAUNCH();
            return RGNN_OK;
        };
        // While there is less than a workgroup of 128 rows for every second compute unit, the wavefronts of a workgroup divide the chunks
        // instead (8000 rows, undivided / divided: d 64, f 256, bf16 10.8 / 8.1 us, fp32 20.7 / 13.0; d 128, f 341, bf16 16.7 / 13.4, 9000 rows, fp32, 45.2 / 32.2).
        constexpr int most = D == 128 ? 2 : 4;           // (four groups' places at width 128 exceed the LDS)
        if (most == 4 && d->rows <= 256 * 32 && a.chunks >= 4) return launch(std::integral_constant<int, most>{});
        if (d->rows <= 256 * 64 && a.chunks >= 2) return launch(std::integral_constant<int, 2>{});
        return launch(std::integral_constant<int, 1>{});
    });
}

rgnn_status_t grad_reduce(const rgnn_ffn_desc_t* d, const FfnGradArgs& k, hipStream_t st) {
    const unsigned blocks = (unsigned)((int64_t)3 * d->width * k.a.chunks * kHid / 64);
    KernelTimer timer(st, "ffn_bwd.reduce");
    if (d->dtype == RGNN_BF16) ffn_grad_reduce_kernel<bf16_t><<<blocks, 256, 0, st>>>(k, d->width);
    else ffn_grad_reduce_kernel<float><<<blocks, 256, 0, st>>>(k, d->width);
    RGNN_CHECK_LAUNCH();
    return RGNN_OK;
}

// dX or the weights' gradients may be null; the other's are the same either way.
rgnn_status_t backward(const rgnn_ffn_desc_t* d, const FfnArgs& a, bool held, void* dX, void* dWg, void* dWu, void* dWd, int accumulate, void* workspace, hipStream_t st) {
    unsigned char* const packed = static_cast<unsigned char*>(workspace);
    const RowsArgs r{a, packed, dX, nullptr, 1, accumulate};
    const FfnGradArgs k{a, reinterpret_cast<float*>(packed + packed_bytes(d, true)), grad_splits(d), ffn_grad_groups(d), dWg, dWu, dWd, accumulate};
    const int rows = dX ? ffn_row_blocks(d) : 0, grads = dWg ? k.splits * k.groups : 0;
    auto run = [&]() -> rgnn_status_t {
        RGNN_DISPATCH_FFN(d, {
            if (rows) RGNN_TRY((launch_pack<D, PL>(a, true, packed, st)));
            constexpr size_t lds = std::max(Weights<D, PL, true>::lds, (size_t)Cut<D, PL>::lds);
            auto* const kernel = held ? ffn_bwd_kernel<D, PL, ACT, true> : ffn_bwd_kernel<D, PL, ACT, false>;
            RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds));
            KernelTimer timer(st, "ffn_bwd");
            kernel<<<rows + grads, 64 * kRowWaves, lds, st>>>(r, k, rows);
            RGNN_CHECK_LAUNCH();
            return RGNN_OK;
        });
    };
    if (rows + grads) RGNN_TRY(run());
    return dWg ? grad_reduce(d, k, st) : RGNN_OK;
}

rgnn_status_t check_desc(const rgnn_ffn_desc_t* d) {
    if (!d) RGNN_FAIL(RGNN_EINVAL, "desc is NULL");
    RGNN_TRY(check_rows(d->rows));
    if (d->rows > kMostRows) RGNN_FAIL(RGNN_EUNSUPPORTED, "rows %lld not supported (up to %lld)", (long long)d->rows, (long long)kMostRows);
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
    const FfnArgs a{desc->rows, desc->hidden, ffn_chunks(desc), X, Wg, Wu, Wd, nullptr, nullptr};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return ffn_few(desc, false) ? ffn_few_fwd(desc, a, out, workspace, st) : forward(desc, a, out, workspace, st);
}

namespace rgnn {
namespace {

// The backward; held: X in 8 bits, given for X.
rgnn_status_t ffn_backward(const rgnn_ffn_desc_t* desc, const void* X, const rgnn_rows8_t* held, const void* Wg, const void* Wu, const void* Wd, const void* dOut,
                           void* dX, void* dWg, void* dWu, void* dWd, void* workspace, void* stream) {
    const bool grads = dWg || dWu || dWd;
    if (grads && !(dWg && dWu && dWd)) RGNN_FAIL(RGNN_EINVAL, "dWg, dWu and dWd are given together or not at all");
    if (!Wg || !Wu || !Wd) RGNN_FAIL(RGNN_EINVAL, "a weight is NULL");
    if (desc->rows > 0 && (!X || !dOut || (held && !held->scales))) RGNN_FAIL(RGNN_EINVAL, "X or dOut is NULL");
    if (!workspace) RGNN_FAIL(RGNN_EWORKSPACE, "workspace is NULL");
    const size_t n = (size_t)desc->rows * desc->width, w = (size_t)desc->hidden * desc->width;
    const int32_t t = desc->dtype;
    const std::initializer_list<Span> written{span(dX, n, t), span(dWg, w, t), span(dWu, w, t), span(dWd, w, t),
                                              Span{static_cast<char*>(workspace), workspace_bytes(desc, true)}};
    RGNN_TRY(check_tensors({held ? code_span(held, desc->rows, desc->width) : span(X, n, t), span(Wg, w, t), span(Wu, w, t), span(Wd, w, t), span(dOut, n, t)}, written));
    if (held)
        for (const Span& s : written)
            if (s.overlaps(scale_span(held, desc->rows, desc->width))) RGNN_FAIL(RGNN_EINVAL, "an output or the workspace overlaps the scales of X");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const FfnArgs a{desc->rows, desc->hidden, ffn_chunks(desc), X, Wg, Wu, Wd, dOut, held ? held->scales : nullptr};
    const int accumulate = (desc->flags & RGNN_FLAG_ACCUMULATE) != 0;
    if (desc->rows > 0 && ffn_few(desc, true)) return ffn_few_bwd(desc, a, held, dX, dWg, dWu, dWd, workspace, st);
    if (desc->rows == 0) dX = nullptr;
    if (!grads || (desc->rows == 0 && accumulate)) dWg = nullptr;
    return backward(desc, a, held, dX, dWg, dWu, dWd, accumulate, workspace, st);
}

}  // namespace
}  // namespace rgnn

extern "C" rgnn_status_t rgnn_ffn_bwd(const rgnn_ffn_desc_t* desc, const void* X, const void* Wg, const void* Wu, const void* Wd, const void* dOut,
                                      void* dX, void* dWg, void* dWu, void* dWd, void* workspace, void* stream) {
    RGNN_TRY(check_desc(desc));
    return ffn_backward(desc, X, nullptr, Wg, Wu, Wd, dOut, dX, dWg, dWu, dWd, workspace, stream);
}

extern "C" rgnn_status_t rgnn_ffn_bwd_rows8(const rgnn_ffn_desc_t* desc, const rgnn_rows8_t* X8, const void* Wg, const void* Wu, const void* Wd, const void* dOut,
                                            void* dX, void* dWg, void* dWu, void* dWd, void* workspace, void* stream) {
    RGNN_TRY(check_desc(desc));
    if (!X8) RGNN_FAIL(RGNN_EINVAL, "X8 is NULL");
    return ffn_backward(desc, X8->codes, X8, Wg, Wu, Wd, dOut, dX, dWg, dWu, dWd, workspace, stream);
}
