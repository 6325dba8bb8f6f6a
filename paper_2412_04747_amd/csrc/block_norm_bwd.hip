// The junction of a block's output with the residual stream, backward: launches, and the sums of the workgroups' partial rows (block_norm_bwd.h has the kernel).
#include "rgnn_internal.h"
#include "device_utils.h"
#include "block_norm_bwd.h"

namespace rgnn {

namespace {

// The workgroups' partial rows, summed in order: a workgroup has kReduceCols columns of all types, which lie together, partial row by partial row.
constexpr int kReduceBlock = 1024;
__global__ __launch_bounds__(kReduceBlock) void block_reduce_kernel(BlockBwdArgs a, int n) {
    __shared__ float4 lds[kReduceBlock];
    const int vectors = (a.p.T + 1) * (kReduceCols / 4), at_once = kReduceBlock / vectors, k = quotient(threadIdx.x, vectors);
    const float4* const part = reinterpret_cast<const float4*>(a.part) + (int64_t)blockIdx.x * n * vectors + threadIdx.x;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float4& o) { v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w; };
    if (k < at_once) {
#pragma unroll 4
        for (int i = k; i < n; i += at_once) add(part[(int64_t)(i - k) * vectors]);
    }
    lds[threadIdx.x] = v;
    for (int h = kReduceBlock / 4; h > 0; h >>= 1) {         // (at_once is a quarter of the threads at most)
        __syncthreads();
        if (k < h && k + h < at_once) {
            add(lds[threadIdx.x + h * vectors]);
            lds[threadIdx.x] = v;
        }
    }
    __syncthreads();
    finish(a, blockIdx.x * kReduceCols, kReduceCols, kReduceBlock, [&](int t, int c) -> float& { return reinterpret_cast<float*>(lds)[t * kReduceCols + c]; });
}

}  // namespace

size_t block_bwd_workspace(const rgnn_block_norm_desc_t* d) {
    return align_up(sizeof(float) * (size_t)std::max(workgroups(d), 1) * (d->types + 1) * part_groups(d->width) * kReduceCols);
}

rgnn_status_t block_bwd(const rgnn_block_norm_desc_t* d, BlockBwdArgs a, bool held, void* workspace, hipStream_t st) {
    a.part = static_cast<float*>(workspace);
    const JunctionPlan p = block_plan(d);
    if (d->rows > 0 && (a.da || a.dstream || a.sums))
        RGNN_TRY(held ? block_bwd_rows8(d, p, a, st) : launch_types<false>(d, p, a, st));
    const int n = workgroups(d);
    if (a.sums && n != 1 && (d->rows > 0 || !a.accumulate)) {
        KernelTimer timer(st, "block_norm_bwd.reduce");
        block_reduce_kernel<<<part_groups(d->width), kReduceBlock, 0, st>>>(a, n);
        RGNN_CHECK_LAUNCH();
    }
    return RGNN_OK;
}

}  // namespace rgnn
