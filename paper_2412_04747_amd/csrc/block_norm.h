// Where a block's output joins the residual stream: what the forward's and the backward's launches share.  Internal.
//
//   n = a q1 w1, q1 = 1 / sqrt(mean(a^2) + eps);   s' = scale[t] s + gate[t] n;   out = s' q2 w2, q2 = 1 / sqrt(mean(s'^2) + eps)
// With g = dOut w2 and dT the whole gradient of s':
//   dT = dSum + q2 (g - s' q2^2 mean(g s')),   dS = scale[t] dT,   h = gate[t] dT w1,   dA = q1 (h - a q1^2 mean(h a))
//   G[t] = sum over the rows of type t of dT a q1:   dgate[t] = w1 G[t],   dw1 = sum over t of gate[t] G[t]
//   dscale[t] = sum over the rows of type t of dT . s,   dw2 = sum over the rows of dOut s' q2
#pragma once
#include "rows8.h"

namespace rgnn {

struct BlockParams {
    const int32_t* types;    // null: one type
    int T;
    const float* w1; const float* gate; const float* scale; const float* w2;
};

struct BlockFwdArgs {
    int64_t rows;
    int width, G;
    float eps;
    BlockParams p;
    const void* a; const void* s;
    void* sum; void* out;
    int8_t* a_codes; uint8_t* a_scales; int8_t* s_codes; uint8_t* s_scales;
};

struct BlockBwdArgs {
    int64_t rows;
    int width, G, accumulate;
    float eps;
    BlockParams p;
    const void* a; const void* s;        // codes, where they are held in 8 bits
    const uint8_t* a_scales; const uint8_t* s_scales;
    const void* dy; const void* ds;
    void* da; void* dstream;
    int sums;                // whether a parameter's gradient is wanted
    float* part;             // [gridDim.x][(T + 1) (width + 1)]: G and dscale of each type, then dw2; of a single workgroup the gradients themselves
    rgnn_block_norm_grads_t grads;
};

// Columns per vector, lanes per row (a workgroup's: kBlock) and vectors per lane: as for the norm, but at most 16 columns per lane.
struct JunctionPlan { int V, G, NV; int64_t turns; };
inline JunctionPlan block_plan(const rgnn_block_norm_desc_t* d) {
    const bool all16 = d->a_dtype == RGNN_BF16 && d->sum_dtype == RGNN_BF16 && d->out_dtype == RGNN_BF16;
    JunctionPlan p;
    p.V = all16 && d->width % 8 == 0 ? 8 : 4;
    const int vectors = (d->width + p.V - 1) / p.V;
    p.G = 1;
    while (p.G < vectors && p.G < 64) p.G *= 2;
    if (vectors > 64 * 16 / p.V) p.G = kBlock;
    p.NV = (vectors + p.G - 1) / p.G;
    p.turns = (d->rows + kBlock / p.G - 1) / (kBlock / p.G);
    return p;
}

// f(vectors' columns, vectors, even) as compile-time values
template <bool ALL16, typename F>
rgnn_status_t block_with_vectors(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, F f) {
    auto count = [&](auto V, auto even) {
        using One = std::integral_constant<int, 1>;
        using Two = std::integral_constant<int, 2>;
        if constexpr (V() == 8) return p.NV <= 1 ? f(V, One{}, even) : f(V, Two{}, even);
        else return p.NV <= 1 ? f(V, One{}, even) : p.NV <= 2 ? f(V, Two{}, even) : f(V, std::integral_constant<int, 4>{}, even);
    };
    if constexpr (ALL16)
        if (p.V == 8) return count(std::integral_constant<int, 8>{}, std::true_type{});
    return d->width % 4 == 0 ? count(std::integral_constant<int, 4>{}, std::true_type{}) : count(std::integral_constant<int, 4>{}, std::false_type{});
}
template <typename F>
rgnn_status_t block_with_types(const rgnn_block_norm_desc_t* d, F f) {
    const float f32 = 0;
    const bf16_t b16 = 0;
    auto third = [&](auto x, auto s) { return d->out_dtype == RGNN_BF16 ? f(x, s, b16) : f(x, s, f32); };
    auto second = [&](auto x) { return d->sum_dtype == RGNN_BF16 ? third(x, b16) : third(x, f32); };
    return d->a_dtype == RGNN_BF16 ? second(b16) : second(f32);
}

// A row's type; negative: it stands for nothing.
__device__ __forceinline__ int row_type(const BlockParams& p, int64_t row, bool live) {
    if (!live) return -1;
    if (!p.types) return 0;
    const int t = p.types[row];
    return (unsigned)t < (unsigned)p.T ? t : -1;
}

size_t block_bwd_workspace(const rgnn_block_norm_desc_t* d);
rgnn_status_t block_bwd_rows8(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, const BlockBwdArgs& a, hipStream_t st);
rgnn_status_t block_bwd(const rgnn_block_norm_desc_t* d, BlockBwdArgs a, bool held, void* workspace, hipStream_t st);

}  // namespace rgnn
