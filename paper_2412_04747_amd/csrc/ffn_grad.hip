// Gated feed-forward block: the gradients of its weights (ffn.h has the formulas).
//
// A wavefront owns MT hidden values: their columns of Wg and Wu and rows of Wd stay in its registers, and so do its columns of the
// three gradients while it walks the rows, 32 at a time.  Of each unit it forms g, u and dh = dOut Wd^T with the rows along the
// accumulator's values, which makes act(g) u, dg and du the second operand of X^T dg, X^T du and dOut^T h as they lie; the first
// is read from the rows' planes in the LDS by the transposing read.  The rows are loaded, split into planes and put there by all four
// wavefronts, one unit ahead.
// g, u and dh are formed a second time (the pass of the rows had them with the hidden values along): three products more of eleven, against
// three tensors of the hidden width written and read, six times the bytes of the row tensors at f = 2 d.
// MT = 32, except for fp32 at width 128, whose three planes of the weights and the gradients of 32 values exceed the registers: 16.
// Rows are divided among workgroups in `splits` interleaved shares; a second launch adds the shares in order.
#include <math.h>

#include "rgnn_internal.h"
#include "device_utils.h"
#include "ffn.h"

namespace rgnn {

namespace {

constexpr int UNIT = 32;

// Hidden values of a wavefront (MT), wavefronts of a workgroup, and wavefronts that share a SIMD.
template <int D, int PL> struct Cut {
    static constexpr bool wide = D == 128 && PL == 3;
    static constexpr int MT = PL == 1 && D < 128 ? 32 : 16;
    static constexpr int waves = MT == 32 || wide ? 4 : 8;
    static constexpr int per_simd = wide ? 1 : 2;
};
struct Sizes { int group, resident; };       // hidden values of a workgroup; workgroups that fill the GPU's 256 compute units
template <int D, int PL> constexpr Sizes sizes_of() { return {Cut<D, PL>::MT * Cut<D, PL>::waves, 256 * 4 * Cut<D, PL>::per_simd / Cut<D, PL>::waves}; }
Sizes sizes(const rgnn_ffn_desc_t* d) {
    if (d->dtype == RGNN_BF16) return d->width == 32 ? sizes_of<32, 1>() : d->width == 64 ? sizes_of<64, 1>() : sizes_of<128, 1>();
    return d->width == 32 ? sizes_of<32, 3>() : d->width == 64 ? sizes_of<64, 3>() : sizes_of<128, 3>();
}
int groups_of(const rgnn_ffn_desc_t* d) { return (d->hidden + sizes(d).group - 1) / sizes(d).group; }

// 16-byte piece c of row r of a plane sits at piece c ^ swizzle(r): 16 consecutive rows' pieces lie in different places modulo 256 bytes,
// and so do the pieces of four rows that the transposing read takes together.
template <int D>
__device__ __forceinline__ int swizzle(int r) {
    constexpr int L = D == 128 ? 0 : D == 64 ? 1 : 2;
    return (((r >> L) & (7 >> L)) << 1) | ((r >> 3) & 1);
}

template <int D, int PL, int ACT>
__global__ __launch_bounds__((64 * Cut<D, PL>::waves), (Cut<D, PL>::per_simd)) void ffn_grad_kernel(FfnGradArgs k) {
    constexpr int MT = Cut<D, PL>::MT, WAVES = Cut<D, PL>::waves;
    using T = typename std::conditional<PL == 1, bf16_t, float>::type;
    using Acc = typename std::conditional<MT == 32, v16f, v4f>::type;
    constexpr int KS = MT == 32 ? 16 : 32;               // contraction of an instruction
    constexpr int S = D / KS, NR = MT == 32 ? 16 : 4, RTS = UNIT / MT, STEPS = UNIT / KS, TILES = D / MT;
    constexpr int PLANE = UNIT * D * 2, BUF = 2 * PL * PLANE;
    // pieces of V columns (16 bytes, or 8 where the unit has fewer than the threads) that a thread loads of either tensor
    constexpr int V = PL == 3 || UNIT * D / 8 < 64 * WAVES ? 4 : 8, PIECES = UNIT * D / V, ITEMS = (PIECES + 64 * WAVES - 1) / (64 * WAVES);
    using Raw = typename std::conditional<sizeof(T) * V == 16, rgnn_v4u, rgnn_v2u>::type;
    extern __shared__ unsigned char lds[];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & (MT - 1), kg = lane / MT;
    const FfnArgs& a = k.a;
    // workgroups of one share of the rows are on one chiplet, whose L2 then holds the rows for all of them
    const int split = (int)(blockIdx.x % 8) + 8 * (int)(blockIdx.x / (8 * k.groups)), group = (int)(blockIdx.x / 8) % k.groups;
    if (split >= k.splits) return;
    const int F = a.hidden, FP = a.chunks * kHid, h = (group * WAVES + wave) * MT + m;
    const bool mine = (group * WAVES + wave) * MT < FP;

    bf16x8 wg[S][PL], wu[S][PL], wd[S][PL];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        float vg[8], vu[8], vd[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = KS * s + 8 * kg + j;
            const bool ok = h < F;
            vg[j] = ok ? widen(static_cast<const T*>(a.Wg)[(size_t)c * F + h]) : 0.f;
            vu[j] = ok ? widen(static_cast<const T*>(a.Wu)[(size_t)c * F + h]) : 0.f;
            vd[j] = ok ? widen(static_cast<const T*>(a.Wd)[(size_t)h * D + c]) : 0.f;
        }
        planes8<PL>(vg, wg[s]);
        planes8<PL>(vu, wu[s]);
        planes8<PL>(vd, wd[s]);
    }
    Acc dwg[TILES], dwu[TILES], dwd[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        clear(dwg[t]);
        clear(dwu[t]);
        clear(dwd[t]);
    }

    const int64_t units = (a.rows + UNIT - 1) / UNIT;
    Raw xr[ITEMS], yr[ITEMS];
    auto load = [&](int64_t u) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = threadIdx.x + i * 64 * WAVES, rr = at / (D / V), c = at % (D / V) * V;
            const int64_t row = u * UNIT + rr;
            xr[i] = yr[i] = Raw{};
            if (at < PIECES && row < a.rows) {
                xr[i] = *reinterpret_cast<const Raw*>(static_cast<const T*>(a.X) + row * D + c);
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
            if constexpr (PL == 1) {
                *reinterpret_cast<Raw*>(p) = xr[i];
                *reinterpret_cast<Raw*>(p + PLANE) = yr[i];
            } else {
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = __uint_as_float(xr[i][e]);
                    v[4 + e] = __uint_as_float(yr[i][e]);
                }
                bf16x8 q[PL];
                planes8<PL>(v, q);
#pragma unroll
                for (int l = 0; l < PL; ++l) {
                    const uint4 w = __builtin_bit_cast(uint4, q[l]);
                    *reinterpret_cast<uint2*>(p + l * PLANE) = make_uint2(w.x, w.y);
                    *reinterpret_cast<uint2*>(p + (PL + l) * PLANE) = make_uint2(w.z, w.w);
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
    auto rows_operand = [&](const unsigned char* buf, int at, int which, int i, int s, bf16x8 (&f)[PL]) {
        const unsigned char* const p = buf + ((at ^ (KS * 2 * s)) + i * MT * 2 * D + which * PL * PLANE);
#pragma unroll
        for (int l = 0; l < PL; ++l) f[l] = *reinterpret_cast<const bf16x8*>(p + l * PLANE);
    };
    // columns MT t + m, the rows in the order of the accumulators' values 8 s ..: rows 16 s + 4 kg .. and 8 further, or 4 kg .. and 16 further
    auto cols_operand = [&](const unsigned char* buf, int at, int which, int t, int s, bf16x8 (&f)[PL]) {
        const int p = (at ^ (MT * 2 * t)) + s * 16 * 2 * D + which * PL * PLANE;
        const int q = (at ^ (MT * 2 * t) ^ (MT == 32 ? 16 : 0)) + s * 16 * 2 * D + which * PL * PLANE + (MT == 32 ? 8 : 16) * 2 * D;
#pragma unroll
        for (int l = 0; l < PL; ++l) f[l] = tr8(buf + p + l * PLANE, buf + q + l * PLANE);
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
                bf16x8 f[PL];
                rows_operand(buf, ra, 0, i, s, f);
                mul_add<PL>(f, wg[s], g[i]);
                mul_add<PL>(f, wu[s], up[i]);
                rows_operand(buf, ra, 1, i, s, f);
                mul_add<PL>(f, wd[s], dh[i]);
            }
        }
        bf16x8 hp[STEPS][PL], gp[STEPS][PL], upp[STEPS][PL];
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
            planes8<PL>(vh, hp[s]);
            planes8<PL>(vg, gp[s]);
            planes8<PL>(vu, upp[s]);
        }
        // Three planes: the unit's products are summed on their own and then added, one rounding at the gradient's magnitude per 32 rows.
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            if constexpr (PL == 1) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    bf16x8 f[PL];
                    cols_operand(buf, ca, 0, t, s, f);
                    mul_add<PL>(f, gp[s], dwg[t]);
                    mul_add<PL>(f, upp[s], dwu[t]);
                    cols_operand(buf, ca, 1, t, s, f);
                    mul_add<PL>(f, hp[s], dwd[t]);
                }
            } else {
                Acc tg, tu, td;
                clear(tg);
                clear(tu);
                clear(td);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    bf16x8 f[PL];
                    cols_operand(buf, ca, 0, t, s, f);
                    mul_add<PL>(f, gp[s], tg);
                    mul_add<PL>(f, upp[s], tu);
                    cols_operand(buf, ca, 1, t, s, f);
                    mul_add<PL>(f, hp[s], td);
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

// The shares' sums: 64 elements of [3][D][FP] per workgroup, four per lane, every 16th share, then the sixteen sums in order.  (A lane that
// took all shares by itself waited for 512 loads in a row at d 32: 122 us, now 8.)
template <typename T>
__global__ __launch_bounds__(256) void ffn_grad_reduce_kernel(const float* part, int splits, int D, int F, int FP, T* dWg, T* dWu, T* dWd, int accumulate) {
    __shared__ float lds[16][64];
    const int64_t n = (int64_t)3 * D * FP, base = (int64_t)blockIdx.x * 64;       // (n is a multiple of 96 * 32)
    const int e4 = (threadIdx.x & 15) * 4, k0 = threadIdx.x >> 4;
    float s[4];
    zero_cols<4>(s);
#pragma unroll 4
    for (int k = k0; k < splits; k += 16) {
        float v[4];
        load_cols<4>(part + k * n + base + e4, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) lds[k0][e4 + e] = s[e];
    __syncthreads();
    if (threadIdx.x >= 64) return;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += lds[k][threadIdx.x];
    const int64_t i = base + threadIdx.x;
    const int h = (int)(i % FP), c = (int)(i / FP) % D, which = (int)(i / FP / D);
    if (h >= F) return;
    T* const to = which == 0 ? dWg + (size_t)c * F + h : which == 1 ? dWu + (size_t)c * F + h : dWd + (size_t)h * D + c;
    *to = narrow<T>(accumulate ? sum + widen(*to) : sum);
}

}  // namespace

// As many shares as fill the GPU once, a multiple of 8 for the chiplets; no more than units.
int ffn_grad_splits(const rgnn_ffn_desc_t* d) {
    const int64_t units = (d->rows + UNIT - 1) / UNIT;
    return (int)std::min<int64_t>(std::max(8, sizes(d).resident / groups_of(d) / 8 * 8), units);
}

rgnn_status_t ffn_grad(const rgnn_ffn_desc_t* d, const FfnArgs& a, float* part, void* dWg, void* dWu, void* dWd, hipStream_t st) {
    FfnGradArgs k{a, part, ffn_grad_splits(d), groups_of(d)};
    if (k.splits > 0) {
        auto run = [&]() -> rgnn_status_t {
            RGNN_DISPATCH_FFN(d, {
                constexpr size_t lds = 2 * 2 * PL * UNIT * D * 2;
                auto* const kernel = ffn_grad_kernel<D, PL, ACT>;
                RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds));
                KernelTimer timer(st, "ffn_bwd_weights");
                kernel<<<(unsigned)((k.splits + 7) / 8 * 8 * k.groups), 64 * Cut<D, PL>::waves, lds, st>>>(k);
                RGNN_CHECK_LAUNCH();
                return RGNN_OK;
            });
        };
        RGNN_TRY(run());
    }
    const int FP = a.chunks * kHid, accumulate = (d->flags & RGNN_FLAG_ACCUMULATE) != 0;
    const unsigned blocks = (unsigned)((int64_t)3 * d->width * FP / 64);
    KernelTimer timer(st, "ffn_bwd_weights.reduce");
    if (d->dtype == RGNN_BF16)
        ffn_grad_reduce_kernel<<<blocks, 256, 0, st>>>(part, k.splits, d->width, d->hidden, FP, static_cast<bf16_t*>(dWg), static_cast<bf16_t*>(dWu), static_cast<bf16_t*>(dWd), accumulate);
    else
        ffn_grad_reduce_kernel<<<blocks, 256, 0, st>>>(part, k.splits, d->width, d->hidden, FP, static_cast<float*>(dWg), static_cast<float*>(dWu), static_cast<float*>(dWd), accumulate);
    RGNN_CHECK_LAUNCH();
    return RGNN_OK;
}

}  // namespace rgnn
