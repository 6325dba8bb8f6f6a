// Gated feed-forward block: what its kernels share.  Internal.
//
//   g = X Wg, u = X Wu, h = act(g) u, out = h Wd
//   dh = dOut Wd^T, du = dh act(g), dg = dh u act'(g), dX = dg Wg^T + du Wu^T, dWg = X^T dg, dWu = X^T du, dWd = h^T dOut
//
// The hidden values of a row are formed 32 at a time in the accumulators of the matrix instructions and go from there into the
// next product: what an instruction leaves in a lane (the values of one column at rows 8 (i / 4) + 4 (lane / 32) + i % 4, i = 0 .. 15)
// is, eight by eight, what the next one reads from that lane, if the other operand takes its hidden indices in the same order.
#pragma once
#include "row_ops.h"

namespace rgnn {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned rgnn_v2u __attribute__((ext_vector_type(2)));

constexpr int kHid = 32;                 // hidden values of a chunk

struct FfnArgs {
    int64_t rows;
    int hidden, chunks;                  // chunks = ceil(hidden / kHid)
    const void* X; const void* Wg; const void* Wu; const void* Wd; const void* dOut;
};

// planes of eight values: PL == 1 rounds to bfloat16; PL == 3 is exact to 24 bits, x = hi + mid + lo (each rounded to nearest even)
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

// c += a b.  Three planes: the six products down to 2^-18 of the largest, small ones first; what is left out is below 2^-26, a quarter
// of a rounding of the fp32 product.
template <int PL, typename Acc>
__device__ __forceinline__ void mul_add(const bf16x8 (&a)[PL], const bf16x8 (&b)[PL], Acc& c) {
    if constexpr (PL == 1) {
        c = mfma(a[0], b[0], c);
    } else {
        c = mfma(a[0], b[2], c);
        c = mfma(a[2], b[0], c);
        c = mfma(a[1], b[1], c);
        c = mfma(a[0], b[1], c);
        c = mfma(a[1], b[0], c);
        c = mfma(a[0], b[0], c);
    }
}
template <typename Acc>
__device__ __forceinline__ void clear(Acc& c) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Acc) / 4); ++i) c[i] = 0.f;
}

// act(g) and its derivative.  silu: g s and s (1 + g (1 - s)), s = 1 / (1 + exp(-g)) by the base-2 exponential and reciprocal
// instructions, each right to one unit in the last place.
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

// Eight consecutive columns of a row, as planes; zeros where !ok.
template <int PL, typename T>
__device__ __forceinline__ void load_planes8(const T* p, bool ok, bf16x8 (&f)[PL]) {
    if constexpr (PL == 1) {
        static_assert(sizeof(T) == 2, "one plane: bfloat16 storage");
        uint4 v = make_uint4(0, 0, 0, 0);
        if (ok) v = *reinterpret_cast<const uint4*>(p);
        f[0] = __builtin_bit_cast(bf16x8, v);
    } else {
        float v[8];
        zero_cols<8>(v);
        if (ok) load_cols<8>(p, v);
        planes8<PL>(v, f);
    }
}

struct FfnGradArgs {
    FfnArgs a;
    float* part;             // [splits][3][D][chunks * kHid]: dWg, dWu and dWd transposed
    int splits, groups;      // workgroups by rows and by hidden values
};
// ffn_grad.hip
int ffn_grad_splits(const rgnn_ffn_desc_t* d);
rgnn_status_t ffn_grad(const rgnn_ffn_desc_t* d, const FfnArgs& a, float* part, void* dWg, void* dWu, void* dWd, hipStream_t st);

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
