// The junction of a block's output with the residual stream, backward: launches, and the sums of the workgroups' partial rows (block_norm_bwd.h has the kernel).
#include "rgnn_internal.h"
#include "device_utils.h"
#include "block_norm_bwd.h"

namespace rgnn {

namespace {

// The workgroups' partial rows, summed in order: eight columns per workgroup, 128 lanes of rows each.
constexpr int kReduceCols = 8, kReduceBlock = 1024;
__global__ __launch_bounds__(kReduceBlock) void block_reduce_kernel(BlockBwdArgs a, int n) {
    extern __shared__ float lds[];           // [T + 1][wavefronts][columns]
    constexpr int W = kReduceBlock / 64;
    const int c = blockIdx.x * kReduceCols + (threadIdx.x & (kReduceCols - 1)), k = threadIdx.x / kReduceCols, T = a.p.T;
    const int64_t each = part_len(T, a.width);
    for (int t = 0; t <= T; ++t) {
        float v = 0.f;
        if (c <= a.width)
            for (int i = k; i < n; i += kReduceBlock / kReduceCols) v += a.part[i * each + t * (a.width + 1) + c];
        for (int o = kReduceCols; o < 64; o <<= 1) v += __shfl_xor(v, o);
        if ((threadIdx.x & 63) < kReduceCols) lds[(t * W + (threadIdx.x >> 6)) * kReduceCols + (threadIdx.x & 63)] = v;
    }
    __syncthreads();
    if (threadIdx.x < kReduceCols && c <= a.width)
        finish(a, c, [&](int t) {
            float v = 0.f;
            for (int w = 0; w < W; ++w) v += lds[(t * W + w) * kReduceCols + threadIdx.x];
            return v;
        });
}

}  // namespace

size_t block_bwd_workspace(const rgnn_block_norm_desc_t* d) {
    return align_up(sizeof(float) * (size_t)std::max(workgroups(d), 1) * part_len(d->types, d->width));
}

rgnn_status_t block_bwd(const rgnn_block_norm_desc_t* d, BlockBwdArgs a, bool held, void* workspace, hipStream_t st) {
    a.part = static_cast<float*>(workspace);
    const JunctionPlan p = block_plan(d);
    if (d->rows > 0 && (a.da || a.dstream || a.sums))
        RGNN_TRY(held ? block_bwd_rows8(d, p, a, st) : launch_types<false>(d, p, a, st));
    const int n = workgroups(d);
    if (a.sums && n != 1 && (d->rows > 0 || !a.accumulate)) {
        const size_t lds = sizeof(float) * (size_t)(d->types + 1) * (kReduceBlock / 64) * kReduceCols;
        RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(block_reduce_kernel), lds));
        KernelTimer timer(st, "block_norm_bwd.reduce");
        block_reduce_kernel<<<(d->width + kReduceCols) / kReduceCols, kReduceBlock, lds, st>>>(a, n);
        RGNN_CHECK_LAUNCH();
    }
    return RGNN_OK;
}

}  // namespace rgnn
