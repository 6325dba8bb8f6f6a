// Gated feed-forward block: what its kernels share.  Internal.
//
//   g = X Wg, u = X Wu, h = act(g) u, out = h Wd
//   dh = dOut Wd^T, du = dh act(g), dg = dh u act'(g), dX = dg Wg^T + du Wu^T, dWg = X^T dg, dWu = X^T du, dWd = h^T dOut
//
// The hidden values of a row are formed 32 at a time in the accumulators of the matrix instructions and go from there into the
// next product: what an instruction leaves in a lane (the values of one column at rows 8 (i / 4) + 4 (lane / 32) + i % 4, i = 0 .. 15)
// is, eight by eight, what the next one reads from that lane, if the other operand takes its hidden indices in the same order.
#pragma once
#include <math.h>

#include "row_ops.h"
#include "rows8.h"

namespace rgnn {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned rgnn_v2u __attribute__((ext_vector_type(2)));

constexpr int kHid = 32;                 // hidden values of a chunk

// Planes in which act(g) u, dg and du enter the next product.  bf16: two, 16 bits.  One would round them to bfloat16 there, an error of 2.3e-3
// in the result where its own rounding makes 1.7e-3; with two the result is the rounded one but for a value in a thousand next to a border.
constexpr int hidden_planes(int planes) { return planes == 1 ? 2 : planes; }

struct FfnArgs {
    int64_t rows;
    int hidden, chunks;                  // chunks = ceil(hidden / kHid)
    const void* X; const void* Wg; const void* Wu; const void* Wd; const void* dOut;
    const uint8_t* x_scales;             // X held in 8 bits: X is its codes
};

// Planes of X: rows held in 8 bits are exact in one.
constexpr int x_planes(int planes, bool held) { return held ? 1 : planes; }

// planes of eight values: PL == 1 rounds to bfloat16; PL == 2 keeps 16 bits, PL == 3 is exact to 24: x = hi + mid + lo (each rounded to nearest even)
template <int PL>
__device__ __forceinline__ void planes8(const float (&x)[8], bf16x8 (&p)[PL]) {
    rgnn_v4u q[PL];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a = x[2 * e], b = x[2 * e + 1];
#pragma unroll
        for (int k = 0; k < PL; ++k) {
            const unsigned w = bf16_pack2(a, b);
            q[k][e] = w;
            if (k + 1 < PL) {
                a -= __uint_as_float(w << 16);
                b -= __uint_as_float(w & 0xFFFF0000u);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < PL; ++k) p[k] = __builtin_bit_cast(bf16x8, q[k]);
}

__device__ __forceinline__ v16f mfma(bf16x8 a, bf16x8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v4f mfma(bf16x8 a, bf16x8 b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// c += a b.  Three planes of both: the six products down to 2^-18 of the largest, small ones first; what is left out is below 2^-26, a quarter
// of a rounding of the fp32 product.  One plane and two: both products.
template <typename Acc>
__device__ __forceinline__ void mul_add(const bf16x8 (&a)[1], const bf16x8 (&b)[1], Acc& c) { c = mfma(a[0], b[0], c); }
template <typename Acc>
__device__ __forceinline__ void mul_add(const bf16x8 (&a)[1], const bf16x8 (&b)[2], Acc& c) { c = mfma(a[0], b[0], mfma(a[0], b[1], c)); }
// (three planes and one that is exact: all three products)
template <typename Acc>
__device__ __forceinline__ void mul_add(const bf16x8 (&a)[3], const bf16x8 (&b)[1], Acc& c) { c = mfma(a[0], b[0], mfma(a[1], b[0], mfma(a[2], b[0], c))); }
template <typename Acc>
__device__ __forceinline__ void mul_add(const bf16x8 (&a)[1], const bf16x8 (&b)[3], Acc& c) { c = mfma(a[0], b[0], mfma(a[0], b[1], mfma(a[0], b[2], c))); }
template <typename Acc>
__device__ __forceinline__ void mul_add(const bf16x8 (&a)[3], const bf16x8 (&b)[3], Acc& c) {
    c = mfma(a[0], b[2], c);
    c = mfma(a[2], b[0], c);
    c = mfma(a[1], b[1], c);
    c = mfma(a[0], b[1], c);
    c = mfma(a[1], b[0], c);
    c = mfma(a[0], b[0], c);
}
template <typename Acc>
__device__ __forceinline__ void clear(Acc& c) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Acc) / 4); ++i) c[i] = 0.f;
}

// act(g) and its derivative.  silu: g s and s (1 + g (1 - s)), s = 1 / (1 + exp(-g)) by the base-2 exponential and reciprocal
// instructions, each right to one unit in the last place.  The exponent, g times a rounded constant, is off by up to |g| units in all, which is what g's
// own rounding moves the exponential by: far out on the negative side s has |g| units less, of a value below exp(-|g|).
template <int ACT>
__device__ __forceinline__ float act(float g) {
    if (ACT == RGNN_ACT_RELU) return g <= 0.f ? 0.f : g;       // (NaN stays)
    return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f));
}
template <int ACT>
__device__ __forceinline__ void act_slope(float g, float& a, float& slope) {
    if (ACT == RGNN_ACT_RELU) {
        a = g <= 0.f ? 0.f : g;
        slope = g > 0.f ? 1.f : 0.f;
        return;
    }
    const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f));
    a = g * s;
    slope = s + a * (1.f - s);
}

// Eight consecutive columns, 16 s + 8 kh and on, of row min(row, rows - 1) as planes; zeros past the last row.  (The load itself is not a
// branch's: a wavefront would wait for each of its loads by itself.)
template <int D, int PL, typename T>
__device__ __forceinline__ void load_planes8(const T* X, int64_t row, int64_t rows, int col, bf16x8 (&f)[PL]) {
    const bool ok = row < rows;
    const T* const p = X + (ok ? row : rows - 1) * D + col;
    if constexpr (PL == 1) {
        static_assert(sizeof(T) == 2, "one plane: bfloat16 storage");
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        f[0] = __builtin_bit_cast(bf16x8, make_uint4(ok ? v.x : 0, ok ? v.y : 0, ok ? v.z : 0, ok ? v.w : 0));
    } else {
        float v[8];
        load_cols<8>(p, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = ok ? v[e] : 0.f;
        planes8<PL>(v, f);
    }
}

// Values of 8 bits as bfloat16, two to a word.
template <int V>
__device__ __forceinline__ void held_words(const CodeWords<V>& w, unsigned scale, unsigned (&q)[V / 2]) {
    float v[V];
    from_codes<V>(w, held_step(scale), v);
#pragma unroll
    for (int e = 0; e < V / 2; ++e) q[e] = bf16_pack2(v[2 * e], v[2 * e + 1]);
}
// The columns of X that load_planes8 takes, from the rows as they are given or from their 8 bits.
template <int D, int PL, bool HELD, typename T, int XP>
__device__ __forceinline__ void load_x8(const FfnArgs& a, int64_t row, int col, bf16x8 (&f)[XP]) {
    if constexpr (HELD) {
        const bool ok = row < a.rows;
        const int64_t at = ok ? row : a.rows - 1;
        CodeWords<8> w;
        load_codes<true, 8>(static_cast<const int8_t*>(a.X) + at * D, col, D, w);
        const unsigned b = a.x_scales[at * (D / kHeldBlock) + col / kHeldBlock];
        unsigned q[4];
        held_words<8>(w, ok ? b : 0, q);
        f[0] = __builtin_bit_cast(bf16x8, make_uint4(q[0], q[1], q[2], q[3]));
    } else {
        load_planes8<D, PL>(static_cast<const T*>(a.X), row, a.rows, col, f);
    }
}

constexpr int kRowWaves = 4;             // wavefronts of a workgroup in the passes of the rows, 32 rows each
constexpr int kFrag = 1024;              // bytes of an operand of a wavefront's instruction

// Sections of a chunk's weights, each D / 16 operands of PL planes.
enum { kGate, kUp, kDown, kOut, kGateBack, kUpBack };
__host__ __device__ constexpr int section(bool backward, int i) { return !backward || i < 2 ? i : i == 2 ? kOut : i == 3 ? kGateBack : kUpBack; }

// A lane's eight values of operand s of a section, from the weights as they are given; zeros past the last hidden value.
template <int D, int PL, int WHAT>
__device__ __forceinline__ void weight_values(const FfnArgs& a, int chunk, int s, int lane, float (&v)[8]) {
    using T = typename std::conditional<PL == 1, bf16_t, float>::type;
    const int m = lane & 31, kh = lane >> 5, F = a.hidden;
    const T* const W = static_cast<const T*>(WHAT == kGate || WHAT == kGateBack ? a.Wg : WHAT == kUp || WHAT == kUpBack ? a.Wu : a.Wd);
    if constexpr (WHAT == kOut) {        // eight columns of a row of Wd
        const int h = chunk * kHid + m;
        load_cols<8>(W + (size_t)min(h, F - 1) * D + 16 * s + 8 * kh, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = h < F ? v[j] : 0.f;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // hidden value, column of the row: 16 s + 8 kh + j of hidden value m; or columns 32 (s / 2) + m, the (s % 2)-th 16 hidden values in
            // the order of an accumulator
            const int h = chunk * kHid + (WHAT == kGate || WHAT == kUp ? m : 16 * (s & 1) + 8 * (j >> 2) + 4 * kh + (j & 3));
            const int c = WHAT == kGate || WHAT == kUp ? 16 * s + 8 * kh + j : 32 * (s >> 1) + m;
            const int at = min(h, F - 1);
            v[j] = widen(W[WHAT == kDown ? (size_t)at * D + c : (size_t)c * F + at]);
            v[j] = h < F ? v[j] : 0.f;
        }
    }
}

template <int PL>
__device__ __forceinline__ void operand(const unsigned char* at, bf16x8 (&f)[PL]) {
#pragma unroll
    for (int k = 0; k < PL; ++k) f[k] = *reinterpret_cast<const bf16x8*>(at + k * kFrag + (threadIdx.x & 63) * 16);
}

struct RowsArgs {
    FfnArgs a;
    const unsigned char* packed;
    void* out;               // rows of the result
    float* part;             // with several splits: [splits][rows][D]
    int splits, accumulate;
};

// The lane's row of the result: tile t holds columns 32 t + 8 q + 4 kh + (0..3) in values 4 q .. 4 q + 3.
template <int D, int PL>
__device__ __forceinline__ void store_result(const RowsArgs& r, int split, int64_t row, int kh, const v16f (&y)[D / 32]) {
    using T = typename std::conditional<PL == 1, bf16_t, float>::type;
    if (row >= r.a.rows) return;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[4] = {y[t][4 * q], y[t][4 * q + 1], y[t][4 * q + 2], y[t][4 * q + 3]};
            const int64_t at = row * D + 32 * t + 8 * q + 4 * kh;
            if (r.splits > 1) {
                store_cols<4>(r.part + (int64_t)split * r.a.rows * D + at, v);
            } else {
                T* const p = static_cast<T*>(r.out) + at;
                if (r.accumulate) {
                    float o[4];
                    load_cols<4>(p, o);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += o[e];
                }
                store_cols<4>(p, v);
            }
        }
}

// Hidden values of a chunk while they are formed: gate, up and (backward) the gradient of their product.
template <bool BWD> struct Hidden { v16f g, u; };
template <> struct Hidden<true> { v16f g, u, dh; };

// Value j of act(g) u; backward: of dg and du.
template <int ACT>
__device__ __forceinline__ void activate(const Hidden<false>& h, int j, float& v, float&) { v = act<ACT>(h.g[j]) * h.u[j]; }
template <int ACT>
__device__ __forceinline__ void activate(const Hidden<true>& h, int j, float& v, float& v2) {
    float a, slope;
    act_slope<ACT>(h.g[j], a, slope);
    v = h.dh[j] * h.u[j] * slope;
    v2 = h.dh[j] * a;
}

// The splits' shares of n elements, added in order.  Four columns per thread.
template <typename T>
__device__ __forceinline__ void combine_block(const float* part, int splits, int64_t n, T* out, int accumulate, int block) {
    const int64_t i = ((int64_t)block * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    float sum[4];
    zero_cols<4>(sum);
#pragma unroll 4
    for (int k = 0; k < splits; ++k) {
        float v[4];
        load_cols<4>(part + k * n + i, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += v[e];
    }
    if (accumulate) {
        float o[4];
        load_cols<4>(out + i, o);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += o[e];
    }
    store_cols<4>(out + i, sum);
}

constexpr int kBlockRows = 32 * kRowWaves;
inline int ffn_chunks(const rgnn_ffn_desc_t* d) { return (d->hidden + kHid - 1) / kHid; }
inline int ffn_row_blocks(const rgnn_ffn_desc_t* d) { return (int)((d->rows + kBlockRows - 1) / kBlockRows); }

// Workgroups that form the weights' gradients, by hidden values.
inline int ffn_grad_groups(const rgnn_ffn_desc_t* d) {
    const int columns = kRowWaves * (d->dtype == RGNN_BF16 && d->width < 128 ? 32 : 16);
    return (d->hidden + columns - 1) / columns;
}

// Shares of the rows for them.  A share costs its sums of 3 d f fp32 written and read, 24 d f bytes at some 5 TB/s; a unit of 32 rows takes a
// workgroup 0.016 d us (fp32: 0.04 d).  With n units the sum of both is least at sqrt(3333 n / f) shares (8333); `most` fill the GPU.
inline int ffn_grad_shares(const rgnn_ffn_desc_t* d, int most) {
    const int64_t units = (d->rows + 31) / 32;
    const double best = sqrt((d->dtype == RGNN_BF16 ? 3333.0 : 8333.0) * (double)units / d->hidden);
    return (int)std::min<int64_t>(std::min<int64_t>(most, units), std::max(1, (int)best));
}

// ffn_few.hip: the same for few rows
bool ffn_few(const rgnn_ffn_desc_t* d, bool backward);
size_t ffn_few_bytes(const rgnn_ffn_desc_t* d, bool backward);
rgnn_status_t ffn_few_fwd(const rgnn_ffn_desc_t* d, const FfnArgs& a, void* out, void* workspace, hipStream_t st);
// held: X in 8 bits
rgnn_status_t ffn_few_bwd(const rgnn_ffn_desc_t* d, const FfnArgs& a, bool held, void* dX, void* dWg, void* dWu, void* dWd, void* workspace, hipStream_t st);

#define RGNN_DISPATCH_FFN(DESC, ...)                                                                                   \
    do {                                                                                                               \
        const rgnn_ffn_desc_t& d_ = *(DESC);                                                                           \
        auto act_ = [&](auto D_, auto PL_) -> rgnn_status_t {                                                          \
            constexpr int D = decltype(D_)::value, PL = decltype(PL_)::value;                                          \
            if (d_.activation == RGNN_ACT_RELU) { constexpr int ACT = RGNN_ACT_RELU; __VA_ARGS__; }                    \
            else { constexpr int ACT = RGNN_ACT_SILU; __VA_ARGS__; }                                                   \
        };                                                                                                             \
        auto type_ = [&](auto D_) -> rgnn_status_t {                                                                   \
            return d_.dtype == RGNN_BF16 ? act_(D_, std::integral_constant<int, 1>{}) : act_(D_, std::integral_constant<int, 3>{}); \
        };                                                                                                             \
        return d_.width == 32 ? type_(std::integral_constant<int, 32>{})                                               \
             : d_.width == 64 ? type_(std::integral_constant<int, 64>{}) : type_(std::integral_constant<int, 128>{});  \
    } while (0)

}  // namespace rgnn
