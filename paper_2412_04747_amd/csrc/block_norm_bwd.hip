// The junction of a block's output with the residual stream, backward: launches, and the sums of the workgroups' partial rows (block_norm_bwd.h has the kernel).
#include "rgnn_internal.h"
#include "device_utils.h"
#include "block_norm_bwd.h"

namespace rgnn {

namespace {

// Sum over a wavefront's lanes of the same parity.
__device__ __forceinline__ float alternate_lanes_sum(float v) {
    v += dpp_move<kDppQuadSwap2>(v);
    v += dpp_move<kDppRowRotate + 4>(v);
    v += dpp_move<kDppRowRotate + 8>(v);
    return rows_sum(v);
}

// The workgroups' partial rows, summed in order: eight columns per workgroup, two lanes for a partial row's, 512 partial rows at a time.
constexpr int kReduceCols = 8, kReduceBlock = 1024, kReduceTypes = 4, kReduceWaves = kReduceBlock / 64;
__global__ __launch_bounds__(kReduceBlock) void block_reduce_kernel(BlockBwdArgs a, int n) {
    extern __shared__ float lds[];           // [T + 1][wavefronts][columns]
    const int half = threadIdx.x & 1, k = threadIdx.x >> 1, wave = threadIdx.x >> 6, T = a.p.T, L = part_len(a.width);
    const int c = min((int)blockIdx.x * kReduceCols + 4 * half, L - 4);
    for (int t0 = 0; t0 <= T; t0 += kReduceTypes) {          // (loads of several types on their way together)
        float4 v[kReduceTypes];
#pragma unroll
        for (int q = 0; q < kReduceTypes; ++q) v[q] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i = k; i < n; i += kReduceBlock / 2)
#pragma unroll
            for (int q = 0; q < kReduceTypes; ++q) {
                const float4 o = *reinterpret_cast<const float4*>(a.part + ((int64_t)i * (T + 1) + min(t0 + q, T)) * L + c);
                v[q].x += o.x; v[q].y += o.y; v[q].z += o.z; v[q].w += o.w;
            }
#pragma unroll
        for (int q = 0; q < kReduceTypes; ++q) {
            if (t0 + q > T) break;
            const float4 sum = make_float4(alternate_lanes_sum(v[q].x), alternate_lanes_sum(v[q].y), alternate_lanes_sum(v[q].z), alternate_lanes_sum(v[q].w));
            if ((threadIdx.x & 63) < 2) *reinterpret_cast<float4*>(lds + ((t0 + q) * kReduceWaves + wave) * kReduceCols + 4 * half) = sum;
        }
    }
    __syncthreads();
    auto at = [&](int t, int c) -> float& { return lds[t * kReduceWaves * kReduceCols + c]; };
    for (int i = threadIdx.x; i < (T + 1) * kReduceCols; i += kReduceBlock) {
        float& sum = at(i / kReduceCols, i % kReduceCols);
#pragma unroll
        for (int w = 1; w < kReduceWaves; ++w) sum += (&sum)[w * kReduceCols];
    }
    __syncthreads();
    finish(a, blockIdx.x * kReduceCols, kReduceCols, kReduceBlock, at);
}

}  // namespace

size_t block_bwd_workspace(const rgnn_block_norm_desc_t* d) {
    return align_up(sizeof(float) * (size_t)std::max(workgroups(d), 1) * (d->types + 1) * part_len(d->width));
}

rgnn_status_t block_bwd(const rgnn_block_norm_desc_t* d, BlockBwdArgs a, bool held, void* workspace, hipStream_t st) {
    a.part = static_cast<float*>(workspace);
    const JunctionPlan p = block_plan(d);
    if (d->rows > 0 && (a.da || a.dstream || a.sums))
        RGNN_TRY(held ? block_bwd_rows8(d, p, a, st) : launch_types<false>(d, p, a, st));
    const int n = workgroups(d);
    if (a.sums && n != 1 && (d->rows > 0 || !a.accumulate)) {
        const size_t lds = sizeof(float) * (size_t)(d->types + 1) * kReduceWaves * kReduceCols;
        RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(block_reduce_kernel), lds));
        KernelTimer timer(st, "block_norm_bwd.reduce");
        block_reduce_kernel<<<(part_len(d->width) + kReduceCols - 1) / kReduceCols, kReduceBlock, lds, st>>>(a, n);
        RGNN_CHECK_LAUNCH();
    }
    return RGNN_OK;
}

}  // namespace rgnn
