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

constexpr int kWaves = 4;
constexpr int UNIT = 32;

// 16-byte piece c of row r of a plane sits at piece c ^ swizzle(r): 16 consecutive rows' pieces lie in different places modulo 256 bytes,
// and so do the pieces of four rows that the transposing read takes together.
template <int D>
__device__ __forceinline__ int swizzle(int r) {
    constexpr int L = D == 128 ? 0 : D == 64 ? 1 : 2;
    return (((r >> L) & (7 >> L)) << 1) | ((r >> 3) & 1);
}

template <int D, int PL, int ACT, int MT>
__global__ __launch_bounds__(64 * kWaves, 1) void ffn_grad_kernel(FfnGradArgs k) {
    using T = typename std::conditional<PL == 1, bf16_t, float>::type;
    using Acc = typename std::conditional<MT == 32, v16f, v4f>::type;
    constexpr int KS = MT == 32 ? 16 : 32;               // contraction of an instruction
    constexpr int S = D / KS, NR = MT == 32 ? 16 : 4, RTS = UNIT / MT, STEPS = UNIT / KS, TILES = D / MT;
    constexpr int PLANE = UNIT * D * 2, BUF = 2 * PL * PLANE;
    constexpr int ITEMS = UNIT * D / 4 / (64 * kWaves);  // pieces of four columns that a thread loads of either tensor
    extern __shared__ unsigned char lds[];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & (MT - 1), kg = lane / MT;
    const FfnArgs& a = k.a;
    // workgroups of one share of the rows are on one chiplet, whose L2 then holds the rows for all of them
    const int split = (int)(blockIdx.x % 8) + 8 * (int)(blockIdx.x / (8 * k.groups)), group = (int)(blockIdx.x / 8) % k.groups;
    if (split >= k.splits) return;
    const int F = a.hidden, FP = a.chunks * kHid, h = (group * kWaves + wave) * MT + m;
    const bool mine = (group * kWaves + wave) * MT < FP;

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
    float xr[ITEMS][4], yr[ITEMS][4];
    auto load = [&](int64_t u) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = threadIdx.x + i * 64 * kWaves, rr = at / (D / 4), c = at % (D / 4) * 4;
            const int64_t row = u * UNIT + rr;
            zero_cols<4>(xr[i]);
            zero_cols<4>(yr[i]);
            if (row < a.rows) {
                load_cols<4>(static_cast<const T*>(a.X) + row * D + c, xr[i]);
                load_cols<4>(static_cast<const T*>(a.dOut) + row * D + c, yr[i]);
            }
        }
    };
    auto put = [&](unsigned char* buf) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = threadIdx.x + i * 64 * kWaves, rr = at / (D / 4), c = at % (D / 4) * 4;
            unsigned char* const p = buf + rr * (2 * D) + (((c >> 3) ^ swizzle<D>(rr)) << 4) + (c & 4) * 2;
            const float v[8] = {xr[i][0], xr[i][1], xr[i][2], xr[i][3], yr[i][0], yr[i][1], yr[i][2], yr[i][3]};
            bf16x8 q[PL];
            planes8<PL>(v, q);
#pragma unroll
            for (int l = 0; l < PL; ++l) {
                const uint4 w = __builtin_bit_cast(uint4, q[l]);
                *reinterpret_cast<uint2*>(p + l * PLANE) = make_uint2(w.x, w.y);
                *reinterpret_cast<uint2*>(p + (PL + l) * PLANE) = make_uint2(w.z, w.w);
            }
        }
    };
    // rows of tile i, columns KS s + 8 kg ..: of X (which = 0) or dOut (1)
    auto rows_operand = [&](const unsigned char* buf, int which, int i, int s, bf16x8 (&f)[PL]) {
        const int r = i * MT + m;
        const unsigned char* const p = buf + which * PL * PLANE + r * (2 * D) + (((KS / 8 * s + kg) ^ swizzle<D>(r)) << 4);
#pragma unroll
        for (int l = 0; l < PL; ++l) f[l] = *reinterpret_cast<const bf16x8*>(p + l * PLANE);
    };
    // columns MT t + m, the rows in the order of the accumulators' values 8 s ..
    const int i16 = lane & 15, half = MT == 32 ? (lane >> 4) & 1 : 0;
    auto cols_operand = [&](const unsigned char* buf, int which, int t, int s, bf16x8 (&f)[PL]) {
        const int r0 = (MT == 32 ? 16 * s : 0) + 4 * kg + (i16 >> 2), r1 = r0 + (MT == 32 ? 8 : 16);
        const int piece = (MT * t + 16 * half) / 8 + ((i16 & 3) >> 1), low = (i16 & 1) * 8;
        const unsigned char* const b = buf + which * PL * PLANE;
        const unsigned char* const p = b + r0 * (2 * D) + ((piece ^ swizzle<D>(r0)) << 4) + low;
        const unsigned char* const q = b + r1 * (2 * D) + ((piece ^ swizzle<D>(r1)) << 4) + low;
#pragma unroll
        for (int l = 0; l < PL; ++l) f[l] = tr8(p + l * PLANE, q + l * PLANE);
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
        Acc g[RTS], up[RTS], dh[RTS];
#pragma unroll
        for (int i = 0; i < RTS; ++i) {
            clear(g[i]);
            clear(up[i]);
            clear(dh[i]);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                bf16x8 f[PL];
                rows_operand(buf, 0, i, s, f);
                mul_add<PL>(f, wg[s], g[i]);
                mul_add<PL>(f, wu[s], up[i]);
                rows_operand(buf, 1, i, s, f);
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
                    cols_operand(buf, 0, t, s, f);
                    mul_add<PL>(f, gp[s], dwg[t]);
                    mul_add<PL>(f, upp[s], dwu[t]);
                    cols_operand(buf, 1, t, s, f);
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
                    cols_operand(buf, 0, t, s, f);
                    mul_add<PL>(f, gp[s], tg);
                    mul_add<PL>(f, upp[s], tu);
                    cols_operand(buf, 1, t, s, f);
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

// The shares' sums, in order: thread per element of [3][D][FP].
template <typename T>
__global__ __launch_bounds__(256) void ffn_grad_reduce_kernel(const float* part, int splits, int D, int F, int FP, T* dWg, T* dWu, T* dWd, int accumulate) {
    const int64_t n = (int64_t)3 * D * FP, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int h = (int)(i % FP), c = (int)(i / FP) % D, which = (int)(i / FP / D);
    if (h >= F) return;
    float s = 0.f;
    for (int k = 0; k < splits; ++k) s += part[k * n + i];
    T* const to = which == 0 ? dWg + (size_t)c * F + h : which == 1 ? dWu + (size_t)c * F + h : dWd + (size_t)h * D + c;
    *to = narrow<T>(accumulate ? s + widen(*to) : s);
}

}  // namespace

static int tile_of(const rgnn_ffn_desc_t* d) { return d->dtype == RGNN_F32 && d->width == 128 ? 16 : 32; }
int ffn_grad_group(const rgnn_ffn_desc_t* d) { return kWaves * tile_of(d); }
// As many shares as make one workgroup per compute unit (two where both fit), a multiple of 8 for the chiplets; no more than units.
int ffn_grad_splits(const rgnn_ffn_desc_t* d) {
    const int64_t units = (d->rows + UNIT - 1) / UNIT;
    const int groups = (d->hidden + ffn_grad_group(d) - 1) / ffn_grad_group(d);
    const int64_t want = std::max(8, 512 / groups / 8 * 8);
    return (int)std::min(want, units);
}

rgnn_status_t ffn_grad(const rgnn_ffn_desc_t* d, const FfnArgs& a, float* part, void* dWg, void* dWu, void* dWd, hipStream_t st) {
    FfnGradArgs k{a, part, ffn_grad_splits(d), (d->hidden + ffn_grad_group(d) - 1) / ffn_grad_group(d)};
    if (k.splits > 0) {
        auto run = [&]() -> rgnn_status_t {
            RGNN_DISPATCH_FFN(d, {
                constexpr int MT = PL == 3 && D == 128 ? 16 : 32;
                constexpr size_t lds = 2 * 2 * PL * UNIT * D * 2;
                auto* const kernel = ffn_grad_kernel<D, PL, ACT, MT>;
                RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds));
                KernelTimer timer(st, "ffn_bwd_weights");
                kernel<<<(unsigned)((k.splits + 7) / 8 * 8 * k.groups), 64 * kWaves, lds, st>>>(k);
                RGNN_CHECK_LAUNCH();
                return RGNN_OK;
            });
        };
        RGNN_TRY(run());
    }
    const int FP = a.chunks * kHid, accumulate = (d->flags & RGNN_FLAG_ACCUMULATE) != 0;
    const unsigned blocks = (unsigned)(((int64_t)3 * d->width * FP + 255) / 256);
    KernelTimer timer(st, "ffn_bwd_weights.reduce");
    if (d->dtype == RGNN_BF16)
        ffn_grad_reduce_kernel<<<blocks, 256, 0, st>>>(part, k.splits, d->width, d->hidden, FP, static_cast<bf16_t*>(dWg), static_cast<bf16_t*>(dWu), static_cast<bf16_t*>(dWd), accumulate);
    else
        ffn_grad_reduce_kernel<<<blocks, 256, 0, st>>>(part, k.splits, d->width, d->hidden, FP, static_cast<float*>(dWg), static_cast<float*>(dWu), static_cast<float*>(dWd), accumulate);
    RGNN_CHECK_LAUNCH();
    return RGNN_OK;
}

}  // namespace rgnn
