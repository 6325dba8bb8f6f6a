// The feed-forward block's pass of the rows over weights that are laid out: a workgroup's work (ffn.hip says how).  Internal.
#pragma once
#include "ffn.h"

namespace rgnn {

// N operands from memory into the LDS, by WAVES wavefronts
template <int N, int WAVES>
__device__ __forceinline__ void fetch(const unsigned char* from, unsigned char* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & (WAVES - 1);
#pragma unroll
    for (int i = 0; i < (N + WAVES - 1) / WAVES; ++i) {
        const int k = i * WAVES + wave;
        if (N % WAVES == 0 || k < N)
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
// the vector unit then work at the same time within a wavefront, which takes the registers of a second set of hidden values).  A second wavefront per
// SIMD is worth more where the registers allow only one of both: backward, 1M rows, d 64, f 256, fp32, this pass 950 us with one wavefront and the
// second set, 855 with two and without.
template <int D, int PL, bool BWD> struct RowsCut {
    static constexpr int per_simd = D == 128 && PL == 3 && BWD ? 1 : 2;
    static constexpr bool ahead = !((BWD && (D == 128 || PL == 3)) || (D == 128 && PL == 3));
    static constexpr int depth = PL == 1 ? (BWD ? 3 : 4) : 2;     // steps of the second products that an operand is read ahead, and one
};

// 128 rows, all chunks.  GROUPS > 1: 128 / GROUPS rows, whose chunks are divided among the groups of wavefronts, each with places in the LDS of its own; the
// shares are added through the LDS, in order.
template <int D, int PL, int ACT, bool BWD, int GROUPS = 1>
__device__ __forceinline__ void rows_block(const RowsArgs& r, int64_t block, unsigned char* lds) {
    using W = Weights<D, PL, BWD>;
    using Cut = RowsCut<D, PL, BWD>;
    constexpr int S = D / 16, TILES = D / 32, HP = hidden_planes(PL);
    using T = typename std::conditional<PL == 1, bf16_t, float>::type;
    constexpr int WAVES = kRowWaves / GROUPS;
    const int wave = (threadIdx.x >> 6) & (WAVES - 1), lane = threadIdx.x & 63, m = lane & 31, kh = lane >> 5;
    const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / WAVES : 0;
    const int64_t row = (block * WAVES + wave) * 32 + m;
    const int c0 = GROUPS > 1 ? r.a.chunks * group / GROUPS : 0, c1 = GROUPS > 1 ? r.a.chunks * (group + 1) / GROUPS : r.a.chunks;
    unsigned char* const mine = lds + group * W::lds;
    auto first = [&](int c) { return mine + (W::twice ? (c & 1) * (W::first + W::second) * kFrag : 0); };
    auto second = [&](int c) { return first(c) + W::first * kFrag; };
    auto fetch_first = [&](int c) { if (c < c1) fetch<W::first, WAVES>(r.packed + (size_t)c * (W::first + W::second) * kFrag, first(c)); };
    auto fetch_second = [&](int c) { if (c < c1) fetch<W::second, WAVES>(r.packed + ((size_t)c * (W::first + W::second) + W::first) * kFrag, second(c)); };
    fetch_first(c0);
    if (W::twice) {
        if (Cut::ahead) fetch_first(c0 + 1);
        fetch_second(c0);
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
    // backward, whose registers are full, is left to it (2M rows, d 128, f 512, bf16, forward: 1061 us without the fences, 1050 with;
    // 200017 rows, f 341, backward: 300 and 306).
    auto fence = [] { if constexpr (!BWD) __builtin_amdgcn_sched_barrier(0); };
    struct FirstOps { bf16x8 f[BWD ? 3 : 2][PL]; };
    struct SecondOps { bf16x8 f[BWD ? 2 : 1][PL]; };
    auto read_first = [&](const unsigned char* w, int s) {
        FirstOps o;
#pragma unroll
        for (int k = 0; k < (BWD ? 3 : 2); ++k) operand(w + (k * S + s) * PL * kFrag, o.f[k]);
        return o;
    };
    // Steps of the second products: tile and half of the chunk's hidden values.  One plane: the first halves of all tiles while the second's values are
    // split; three: a tile's halves after each other, whose products are summed on their own and then added, one rounding at the result's magnitude per
    // 32 hidden values instead of twelve (1M rows, d 64, f 256, error of dX against 64 bits 3.9e-7 before; f 16384 2.8e-6).
    constexpr bool OWN = PL == 3;
    auto tile = [](int q) { return OWN ? q / 2 : q % TILES; };
    auto part = [](int q) { return OWN ? q % 2 : q / TILES; };
    auto read_second = [&](const unsigned char* w, int q) {
        SecondOps o;
#pragma unroll
        for (int k = 0; k < (BWD ? 2 : 1); ++k) operand(w + (k * S + 2 * tile(q) + part(q)) * PL * kFrag, o.f[k]);
        return o;
    };
    // the s-th sixteen columns' share of the chunk's hidden values
    auto form = [&](const FirstOps& o, int s, Hidden<BWD>& h) {
        mul_add(o.f[0], x[s], h.g);
        mul_add(o.f[1], x[s], h.u);
        if constexpr (BWD) mul_add(o.f[2], dy[s], h.dh);
    };
    // Chunk c's share of the result, from act(g) u (dg and du) in v (and v2).  o: operands of the first steps, on their way already.
    constexpr int DEPTH = Cut::depth < S ? Cut::depth : S;
    auto result = [&](int c, SecondOps (&o)[DEPTH], const float (&v)[16], const float (&v2)[16]) {
        bf16x8 p[2][HP], p2[2][HP];
        auto round = [&](int s) {
            planes8<HP>(*reinterpret_cast<const float(*)[8]>(v + 8 * s), p[s]);
            if constexpr (BWD) planes8<HP>(*reinterpret_cast<const float(*)[8]>(v2 + 8 * s), p2[s]);
        };
        // (forward, the previous tile's is added while this one's instructions run; the backward has no registers left for a second)
        constexpr int OWNS = BWD ? 1 : 2;
        v16f own[OWNS];
        auto add = [&](int t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) y[t][i] += own[t % OWNS][i];
        };
        round(0);
#pragma unroll
        for (int q = 0; q < S; ++q) {
            if (q + DEPTH - 1 < S) o[(q + DEPTH - 1) % DEPTH] = read_second(second(c), q + DEPTH - 1);
            fence();
            const int s = part(q), t = tile(q);
            if (OWN && s == 0) clear(own[t % OWNS]);
            v16f& to = OWN ? own[t % OWNS] : y[t];
            mul_add(o[q % DEPTH].f[0], p[s], to);
            if constexpr (BWD) mul_add(o[q % DEPTH].f[1], p2[s], to);
            if (q == 0) round(1);
            if (OWN && OWNS == 1 && s == 1) add(t);
            if (OWN && OWNS == 2 && s == 0 && t > 0) add(t - 1);
            fence();
        }
        if (OWN && OWNS == 2) add(TILES - 1);
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
        for (int s = 0; s < S; ++s) form(read_first(first(c0), s), s, a);
        if (!W::twice) {
            __syncthreads();
            fetch_first(c0 + 1);
        }
        // (two at a time: the sets of hidden values change places without being moved)
        constexpr std::true_type more;
        constexpr std::false_type last;
        int c = c0;
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
        for (int c = c0; c < c1; ++c) {
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
    if constexpr (GROUPS > 1) {
        // the groups' numbers of chunks differ by one at most: as many barriers for all
        if (c1 - c0 < (r.a.chunks + GROUPS - 1) / GROUPS) {
            arrived();
            if (!W::twice) arrived();
        }
        static_assert((GROUPS - 1) * WAVES * TILES * 16 * 256 <= GROUPS * W::lds, "the shares fit the weights' places");
        auto share = [&](int g) { return reinterpret_cast<float*>(lds) + ((g - 1) * WAVES + wave) * TILES * 16 * 64 + lane; };
        __syncthreads();
        if (group > 0) {
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) share(group)[(t * 16 + i) * 64] = y[t][i];
        }
        __syncthreads();
        if (group > 0) return;
        for (int g = 1; g < GROUPS; ++g)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) y[t][i] += share(g)[(t * 16 + i) * 64];
    }
    store_result<D, PL>(r, 0, row, kh, y);
}

}  // namespace rgnn
