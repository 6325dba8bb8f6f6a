// The gradients of the feed-forward block's weights: a workgroup's work.  Internal.
//
// A wavefront owns MT hidden values: their columns of Wg and Wu and rows of Wd stay in its registers, and so do its columns of the
// three gradients while it walks the rows, 32 at a time.  Of each unit it forms g, u and dh = dOut Wd^T with the rows along the
// accumulator's values, which makes act(g) u, dg and du the second operand of X^T dg, X^T du and dOut^T h as they lie; the first
// is read from the rows' planes in the LDS by the transposing read.  The rows are loaded, split into planes and put there by all
// wavefronts of the workgroup, one unit ahead.
// g, u and dh are formed a second time (the pass of the rows has them with the hidden values along): three products more of eleven, against
// three tensors of the hidden width written and read, six times the bytes of the row tensors at f = 2 d.
// MT = 32 for bf16 up to width 64 (1M rows, d 64, f 256, this pass alone: 320 us, 344 with 16); 16 otherwise, where 32 exceed the registers that leave two
// wavefronts per SIMD (fp32, the same size: 977 us, 1965 with 32; bf16, 200017 rows, d 128, f 341: 178 and 1254).
// Rows are divided among workgroups in interleaved shares, which another launch adds in order.
#pragma once
#include "ffn.h"

namespace rgnn {

constexpr int UNIT = 32;

template <int D, int PL> struct Cut {
    static constexpr int MT = PL == 1 && D < 128 ? 32 : 16;      // hidden values of a wavefront
    static constexpr int lds = 2 * 2 * PL * UNIT * D * 2;        // two units of either tensor (of held rows in fp32 a third is left over)
};
struct FfnGradArgs {
    FfnArgs a;
    float* part;             // [splits][3][D][chunks * kHid]: dWg, dWu and dWd transposed
    int splits, groups;      // workgroups by rows and by hidden values
    void* dWg; void* dWu; void* dWd;     // with one split: the results themselves
    int accumulate;
};
// 16-byte piece c of row r of a plane sits at piece c ^ swizzle(r): 16 consecutive rows' pieces lie in different places modulo 256 bytes,
// and so do the pieces of four rows that the transposing read takes together.
template <int D>
__device__ __forceinline__ int swizzle(int r) {
    constexpr int L = D == 128 ? 0 : D == 64 ? 1 : 2;
    return (((r >> L) & (7 >> L)) << 1) | ((r >> 3) & 1);
}

// The workgroup's share of the rows, `split`, and of the hidden values, `group`.
template <int D, int PL, int ACT, bool DIRECT, bool HELD = false>
__device__ __forceinline__ void grad_block(const FfnGradArgs& k, int split, int group, unsigned char* lds) {
    constexpr int MT = Cut<D, PL>::MT, WAVES = kRowWaves, HP = hidden_planes(PL), XP = x_planes(PL, HELD);
    using T = typename std::conditional<PL == 1, bf16_t, float>::type;
    using Acc = typename std::conditional<MT == 32, v16f, v4f>::type;
    constexpr int KS = MT == 32 ? 16 : 32;               // contraction of an instruction
    constexpr int S = D / KS, NR = MT == 32 ? 16 : 4, RTS = UNIT / MT, STEPS = UNIT / KS, TILES = D / MT;
    constexpr int PLANE = UNIT * D * 2, BUF = (XP + PL) * PLANE;
    // pieces of V columns (16 bytes, or 8 where the unit has fewer than the threads) that a thread loads of either tensor
    constexpr int V = PL == 3 || UNIT * D / 8 < 64 * WAVES ? 4 : 8, PIECES = UNIT * D / V, ITEMS = (PIECES + 64 * WAVES - 1) / (64 * WAVES);
    using Raw = typename std::conditional<sizeof(T) * V == 16, rgnn_v4u, rgnn_v2u>::type;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & (MT - 1), kg = lane / MT;
    const FfnArgs& a = k.a;
    const int F = a.hidden, FP = a.chunks * kHid, h = (group * WAVES + wave) * MT + m;
    const bool mine = (group * WAVES + wave) * MT < F;       // (what a chunk's end leaves in `part` is read by nobody)

    bf16x8 wg[S][PL], wu[S][PL], wd[S][PL];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        float vg[8], vu[8];
        const bool ok = h < F;
        const int hh = min(h, F - 1);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const size_t at = (size_t)(KS * s + 8 * kg + j) * F + hh;
            vg[j] = widen(static_cast<const T*>(a.Wg)[at]);
            vu[j] = widen(static_cast<const T*>(a.Wu)[at]);
            vg[j] = ok ? vg[j] : 0.f;
            vu[j] = ok ? vu[j] : 0.f;
        }
        planes8<PL>(vg, wg[s]);
        planes8<PL>(vu, wu[s]);
        load_planes8<D, PL>(static_cast<const T*>(a.Wd), h, F, KS * s + 8 * kg, wd[s]);
    }
    Acc dwg[TILES], dwu[TILES], dwd[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        clear(dwg[t]);
        clear(dwu[t]);
        clear(dwd[t]);
    }

    const int64_t units = (a.rows + UNIT - 1) / UNIT;
    Raw xr[HELD ? 1 : ITEMS], yr[ITEMS];
    CodeWords<V> codes[HELD ? ITEMS : 1];
    unsigned scales[HELD ? ITEMS : 1];
    auto load = [&](int64_t u) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = threadIdx.x + i * 64 * WAVES, rr = at / (D / V), c = at % (D / V) * V;
            const int64_t row = u * UNIT + rr;
            yr[i] = Raw{};
            if constexpr (HELD) {
                scales[i] = 0;
#pragma unroll
                for (int q = 0; q < V / 4; ++q) codes[i][q] = 0;
            } else {
                xr[i] = Raw{};
            }
            if (at < PIECES && row < a.rows) {
                if constexpr (HELD) {
                    load_codes<true, V>(static_cast<const int8_t*>(a.X) + row * D, c, D, codes[i]);
                    scales[i] = a.x_scales[row * (D / kHeldBlock) + c / kHeldBlock];
                } else {
                    xr[i] = *reinterpret_cast<const Raw*>(static_cast<const T*>(a.X) + row * D + c);
                }
                yr[i] = *reinterpret_cast<const Raw*>(static_cast<const T*>(a.dOut) + row * D + c);
            }
        }
    };
    auto put = [&](unsigned char* buf) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = threadIdx.x + i * 64 * WAVES, rr = at / (D / V), c = at % (D / V) * V;
            if (PIECES % (64 * WAVES) && at >= PIECES) break;
            unsigned char* const p = buf + rr * (2 * D) + (((c >> 3) ^ swizzle<D>(rr)) << 4) + (c & 4) * 2;
            if constexpr (HELD) {
                unsigned q[V / 2];
                held_words<V>(codes[i], scales[i], q);
                __builtin_memcpy(__builtin_assume_aligned(p, 2 * V), q, sizeof(q));
            }
            if constexpr (PL == 1) {
                if constexpr (!HELD) *reinterpret_cast<Raw*>(p) = xr[i];
                *reinterpret_cast<Raw*>(p + PLANE) = yr[i];
            } else {
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = HELD ? 0.f : __uint_as_float(xr[HELD ? 0 : i][e]);
                    v[4 + e] = __uint_as_float(yr[i][e]);
                }
                bf16x8 q[PL];
                planes8<PL>(v, q);
#pragma unroll
                for (int l = 0; l < PL; ++l) {
                    const uint4 w = __builtin_bit_cast(uint4, q[l]);
                    if constexpr (!HELD) *reinterpret_cast<uint2*>(p + l * PLANE) = make_uint2(w.x, w.y);
                    *reinterpret_cast<uint2*>(p + (XP + l) * PLANE) = make_uint2(w.z, w.w);
                }
            }
        }
    };
    // A lane's place in the LDS for the first operand of either kind.  The others are XORs and sums of it with constants, as the swizzle
    // repeats after 16 rows and moves by one piece after 8.
    const int i16 = lane & 15, half = MT == 32 ? (lane >> 4) & 1 : 0, tr = 4 * kg + (i16 >> 2);
    const int rows_at = m * (2 * D) + ((kg ^ swizzle<D>(m)) << 4);
    const int cols_at = (tr & 15) * (2 * D) + (((2 * half + ((i16 & 3) >> 1)) ^ swizzle<D>(tr)) << 4) + (i16 & 1) * 8;
    // rows of tile i, columns KS s + 8 kg ..: of X (which = 0) or dOut (1)
    auto rows_operand = [&](const unsigned char* buf, int at, int which, int i, int s, auto& f) {
        const unsigned char* const p = buf + ((at ^ (KS * 2 * s)) + i * MT * 2 * D + which * XP * PLANE);
#pragma unroll
        for (int l = 0; l < (int)(sizeof(f) / 16); ++l) f[l] = *reinterpret_cast<const bf16x8*>(p + l * PLANE);
    };
    // columns MT t + m, the rows in the order of the accumulators' values 8 s ..: rows 16 s + 4 kg .. and 8 further, or 4 kg .. and 16 further
    auto cols_operand = [&](const unsigned char* buf, int at, int which, int t, int s, auto& f) {
        const int p = (at ^ (MT * 2 * t)) + s * 16 * 2 * D + which * XP * PLANE;
        const int q = (at ^ (MT * 2 * t) ^ (MT == 32 ? 16 : 0)) + s * 16 * 2 * D + which * XP * PLANE + (MT == 32 ? 8 : 16) * 2 * D;
#pragma unroll
        for (int l = 0; l < (int)(sizeof(f) / 16); ++l) f[l] = tr8(buf + p + l * PLANE, buf + q + l * PLANE);
    };

    int64_t u = split;
    if (u < units) load(u);
    int turn = 0;
    for (; u < units; u += k.splits, turn ^= 1) {
        unsigned char* const buf = lds + turn * BUF;
        put(buf);
        if (u + k.splits < units) load(u + k.splits);
        __syncthreads();         // (a wavefront is at most one unit ahead of another: two buffers are enough)
        if (!mine) continue;
        int ra = rows_at, ca = cols_at;
        asm volatile("" : "+v"(ra), "+v"(ca));           // (the places are formed here, not kept across the loop)
        Acc g[RTS], up[RTS], dh[RTS];
#pragma unroll
        for (int i = 0; i < RTS; ++i) {
            clear(g[i]);
            clear(up[i]);
            clear(dh[i]);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                bf16x8 x[XP], f[PL];
                rows_operand(buf, ra, 0, i, s, x);
                mul_add(x, wg[s], g[i]);
                mul_add(x, wu[s], up[i]);
                rows_operand(buf, ra, 1, i, s, f);
                mul_add(f, wd[s], dh[i]);
            }
        }
        bf16x8 hp[STEPS][HP], gp[STEPS][HP], upp[STEPS][HP];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            float vh[8], vg[8], vu[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int v = 8 * s + j, i = v / NR, e = v % NR;
                float av, slope;
                act_slope<ACT>(g[i][e], av, slope);
                vh[j] = av * up[i][e];
                vg[j] = dh[i][e] * up[i][e] * slope;
                vu[j] = dh[i][e] * av;
            }
            planes8<HP>(vh, hp[s]);
            planes8<HP>(vg, gp[s]);
            planes8<HP>(vu, upp[s]);
        }
        // Three planes: the unit's products are summed on their own and then added, one rounding at the gradient's magnitude per 32 rows.
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            if constexpr (PL == 1) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    bf16x8 x[XP], f[PL];
                    cols_operand(buf, ca, 0, t, s, x);
                    mul_add(x, gp[s], dwg[t]);
                    mul_add(x, upp[s], dwu[t]);
                    cols_operand(buf, ca, 1, t, s, f);
                    mul_add(f, hp[s], dwd[t]);
                }
            } else {
                Acc tg, tu, td;
                clear(tg);
                clear(tu);
                clear(td);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    bf16x8 x[XP], f[PL];
                    cols_operand(buf, ca, 0, t, s, x);
                    mul_add(x, gp[s], tg);
                    mul_add(x, upp[s], tu);
                    cols_operand(buf, ca, 1, t, s, f);
                    mul_add(f, hp[s], td);
                }
#pragma unroll
                for (int e = 0; e < NR; ++e) {
                    dwg[t][e] += tg[e];
                    dwu[t][e] += tu[e];
                    dwd[t][e] += td[e];
                }
            }
        }
    }
    if (!mine) return;
    // value e of tile t: column MT t + 8 (e / 4) + 4 kg + e % 4 (MT = 16: 4 kg + e), hidden value h
    if constexpr (DIRECT) {
        if (h >= F) return;
        auto give = [&](void* to, size_t at, float v) {
            T* const p = static_cast<T*>(to) + at;
            *p = narrow<T>(k.accumulate ? v + widen(*p) : v);
        };
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int e = 0; e < NR; ++e) {
                const size_t c = MT * t + (MT == 32 ? 8 * (e >> 2) : 0) + 4 * kg + (e & 3);
                give(k.dWg, c * F + h, dwg[t][e]);
                give(k.dWu, c * F + h, dwu[t][e]);
                give(k.dWd, (size_t)h * D + c, dwd[t][e]);
            }
    } else {
        float* const part = k.part + (size_t)split * 3 * D * FP + h;
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int e = 0; e < NR; ++e) {
                const size_t c = MT * t + (MT == 32 ? 8 * (e >> 2) : 0) + 4 * kg + (e & 3);
                part[c * FP] = dwg[t][e];
                part[(D + c) * FP] = dwu[t][e];
                part[(2 * D + c) * FP] = dwd[t][e];
            }
    }
}

// The shares' sums: 64 elements of [3][D][FP] per workgroup, four per lane, every 16th share, then the sixteen sums in order.  (A lane that
// took all shares by itself waited for 512 loads in a row at d 32: 122 us, now 8.)
template <typename T>
__device__ __forceinline__ void grad_reduce_block(const FfnGradArgs& k, int D, int block, float (&lds)[16][64]) {
    const int F = k.a.hidden, FP = k.a.chunks * kHid;
    const int64_t n = (int64_t)3 * D * FP, base = (int64_t)block * 64;       // (n is a multiple of 96 * 32)
    const int e4 = (threadIdx.x & 15) * 4, k0 = threadIdx.x >> 4;
    float s[4];
    zero_cols<4>(s);
#pragma unroll 4
    for (int i = k0; i < k.splits; i += 16) {
        float v[4];
        load_cols<4>(k.part + i * n + base + e4, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) lds[k0][e4 + e] = s[e];
    __syncthreads();
    if (threadIdx.x >= 64) return;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += lds[i][threadIdx.x];
    const int64_t i = base + threadIdx.x;
    const int h = (int)(i % FP), c = (int)(i / FP) % D, which = (int)(i / FP / D);
    if (h >= F) return;
    T* const to = static_cast<T*>(which == 0 ? k.dWg : which == 1 ? k.dWu : k.dWd) + (which < 2 ? (size_t)c * F + h : (size_t)h * D + c);
    *to = narrow<T>(k.accumulate ? sum + widen(*to) : sum);
}

}  // namespace rgnn
