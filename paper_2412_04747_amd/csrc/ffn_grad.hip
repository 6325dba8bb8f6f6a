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
#include "ffn_grad.h"

namespace rgnn {

namespace {

struct Sizes { int group, resident; };       // hidden values of a workgroup; workgroups that fill the GPU's 256 compute units
template <int D, int PL> constexpr Sizes sizes_of() { return {Cut<D, PL>::MT * Cut<D, PL>::waves, 256 * 4 * Cut<D, PL>::per_simd / Cut<D, PL>::waves}; }
Sizes sizes(const rgnn_ffn_desc_t* d) {
    if (d->dtype == RGNN_BF16) return d->width == 32 ? sizes_of<32, 1>() : d->width == 64 ? sizes_of<64, 1>() : sizes_of<128, 1>();
    return d->width == 32 ? sizes_of<32, 3>() : d->width == 64 ? sizes_of<64, 3>() : sizes_of<128, 3>();
}
int groups_of(const rgnn_ffn_desc_t* d) { return (d->hidden + sizes(d).group - 1) / sizes(d).group; }

template <int D, int PL, int ACT>
__global__ __launch_bounds__((64 * Cut<D, PL>::waves), (Cut<D, PL>::per_simd)) void ffn_grad_kernel(FfnGradArgs k) {
    extern __shared__ unsigned char lds[];
    // workgroups of one share of the rows are on one chiplet, whose L2 then holds the rows for all of them
    const int split = (int)(blockIdx.x % 8) + 8 * (int)(blockIdx.x / (8 * k.groups)), group = (int)(blockIdx.x / 8) % k.groups;
    if (split < k.splits) grad_block<D, PL, ACT, Cut<D, PL>::waves, false>(k, split, group, lds);
}

template <typename T>
__global__ __launch_bounds__(256) void ffn_grad_reduce_kernel(FfnGradArgs k, int D) {
    __shared__ float lds[16][64];
    grad_reduce_block<T>(k, D, blockIdx.x, lds);
}

}  // namespace

// As many shares as fill the GPU once, a multiple of 8 for the chiplets; no more than units.
int ffn_grad_splits(const rgnn_ffn_desc_t* d) {
    const int64_t units = (d->rows + UNIT - 1) / UNIT;
    return (int)std::min<int64_t>(std::max(8, sizes(d).resident / groups_of(d) / 8 * 8), units);
}

rgnn_status_t ffn_grad_reduce(const rgnn_ffn_desc_t* d, const FfnGradArgs& k, hipStream_t st) {
    const unsigned blocks = (unsigned)((int64_t)3 * d->width * k.a.chunks * kHid / 64);
    KernelTimer timer(st, "ffn_bwd_weights.reduce");
    if (d->dtype == RGNN_BF16) ffn_grad_reduce_kernel<bf16_t><<<blocks, 256, 0, st>>>(k, d->width);
    else ffn_grad_reduce_kernel<float><<<blocks, 256, 0, st>>>(k, d->width);
    RGNN_CHECK_LAUNCH();
    return RGNN_OK;
}

rgnn_status_t ffn_grad(const rgnn_ffn_desc_t* d, const FfnArgs& a, float* part, void* dWg, void* dWu, void* dWd, hipStream_t st) {
    const FfnGradArgs k{a, part, ffn_grad_splits(d), groups_of(d), dWg, dWu, dWd, (d->flags & RGNN_FLAG_ACCUMULATE) != 0};
    if (k.splits > 0) {
        auto run = [&]() -> rgnn_status_t {
            RGNN_DISPATCH_FFN(d, {
                constexpr size_t lds = Cut<D, PL>::lds;
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
    return ffn_grad_reduce(d, k, st);
}

}  // namespace rgnn
