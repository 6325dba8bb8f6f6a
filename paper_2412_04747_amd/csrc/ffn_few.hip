// Gated feed-forward block for few rows, where launches and their latency are the time.
//
// The weights are read as they are given and put into the LDS as operands by the workgroups that use them, so that no launch lays them out first;
// the backward's two passes share a launch, some of its workgroups forming dX and the others the weights' gradients; and what several
// workgroups add up is summed by one launch for both.  A call is two launches, or one where nothing is divided.  1000 rows, d 64, f 256, bf16, backward:
// 13.5 us, 19 over weights that a launch laid out.
// ffn_few says which calls are such.
#include <math.h>

#include "rgnn_internal.h"
#include "device_utils.h"
#include "ffn_grad.h"

namespace rgnn {

namespace {

template <int D, int PL, bool BWD> constexpr int rows_lds() { return (BWD ? 5 : 3) * (D / 16) * PL * kFrag; }

// 128 rows, a share of the chunks.
template <int D, int PL, int ACT, bool BWD>
__device__ __forceinline__ void few_rows_block(const RowsArgs& r, int block, int split, unsigned char* lds) {
    constexpr int S = D / 16, TILES = D / 32, SECTIONS = BWD ? 5 : 3, EACH = (S + kRowWaves - 1) / kRowWaves, HP = hidden_planes(PL);
    using T = typename std::conditional<PL == 1, bf16_t, float>::type;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, m = lane & 31, kh = lane >> 5;
    const int64_t row0 = ((int64_t)block * kRowWaves + wave) * 32, row = row0 + m;
    const int c0 = (int)((int64_t)r.a.chunks * split / r.splits), c1 = (int)((int64_t)r.a.chunks * (split + 1) / r.splits);
    bf16x8 x[S][PL], dy[BWD ? S : 1][PL];
    v16f y[TILES];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        load_planes8<D, PL>(static_cast<const T*>(r.a.X), row, r.a.rows, 16 * s + 8 * kh, x[s]);
        if constexpr (BWD) load_planes8<D, PL>(static_cast<const T*>(r.a.dOut), row, r.a.rows, 16 * s + 8 * kh, dy[s]);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) clear(y[t]);
    for (int c = c0; c < c1; ++c) {
        // all loads, then all conversions: the wavefronts wait for memory once per chunk
        float v[SECTIONS][EACH][8];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int s = i * kRowWaves + wave;
            if (S % kRowWaves && s >= S) break;
            weight_values<D, PL, section(BWD, 0)>(r.a, c, s, lane, v[0][i]);
            weight_values<D, PL, section(BWD, 1)>(r.a, c, s, lane, v[1][i]);
            weight_values<D, PL, section(BWD, 2)>(r.a, c, s, lane, v[2][i]);
            if constexpr (BWD) {
                weight_values<D, PL, section(BWD, 3)>(r.a, c, s, lane, v[3][i]);
                weight_values<D, PL, section(BWD, 4)>(r.a, c, s, lane, v[4][i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (c > c0) __syncthreads();
#pragma unroll
        for (int k = 0; k < SECTIONS; ++k)
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int s = i * kRowWaves + wave;
                if (S % kRowWaves && s >= S) break;
                bf16x8 f[PL];
                planes8<PL>(v[k][i], f);
#pragma unroll
                for (int l = 0; l < PL; ++l) *reinterpret_cast<bf16x8*>(lds + ((k * S + s) * PL + l) * kFrag + lane * 16) = f[l];
            }
        __syncthreads();
        if (row0 >= r.a.rows) continue;
        Hidden<BWD> h;
        clear(h.g);
        clear(h.u);
        if constexpr (BWD) clear(h.dh);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            bf16x8 f[PL];
            operand(lds + s * PL * kFrag, f);
            mul_add(f, x[s], h.g);
            operand(lds + (S + s) * PL * kFrag, f);
            mul_add(f, x[s], h.u);
            if constexpr (BWD) {
                operand(lds + (2 * S + s) * PL * kFrag, f);
                mul_add(f, dy[s], h.dh);
            }
        }
        const unsigned char* const w = lds + (BWD ? 3 : 2) * S * PL * kFrag;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            float v[8], v2[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) activate<ACT>(h, 8 * s + j, v[j], v2[j]);
            bf16x8 p[HP], p2[HP], f[PL];
            planes8<HP>(v, p);
            if constexpr (BWD) planes8<HP>(v2, p2);
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                operand(w + (2 * t + s) * PL * kFrag, f);
                mul_add(f, p, y[t]);
                if constexpr (BWD) {
                    operand(w + (S + 2 * t + s) * PL * kFrag, f);
                    mul_add(f, p2, y[t]);
                }
            }
        }
    }
    store_result<D, PL>(r, split, row, kh, y);
}

template <int D, int PL, int ACT>
__global__ __launch_bounds__(64 * kRowWaves, 1) void ffn_few_fwd_kernel(RowsArgs r) {
    extern __shared__ unsigned char lds[];
    few_rows_block<D, PL, ACT, false>(r, blockIdx.x, blockIdx.y, lds);
}

// One row, or up to four in fp32, forward: no matrix instructions, whose 32 rows would be padding.  A workgroup takes 32 hidden values at a time: its lanes read 32
// consecutive ones of a row of Wg and Wu, eight ranges of the columns beside each other, and then rows of Wd, every weight once and coalesced; sums meet in the
// LDS.  (One row, d 128, f 512, fp32: 10.4 us in the kernel above, 6.1 here.)
template <int D, typename T, int ACT, int R>
__global__ __launch_bounds__(256) void ffn_single_fwd_kernel(RowsArgs r) {
    constexpr int KG = 8, K = D / KG, HG = 256 / D, H = kHid / HG;
    __shared__ float x[R][D], part[KG][R][2][kHid], hid[R][kHid], sums[HG][R][D];
    const int t = threadIdx.x, F = r.a.hidden;
    const T* const Wg = static_cast<const T*>(r.a.Wg);
    const T* const Wu = static_cast<const T*>(r.a.Wu);
    const T* const Wd = static_cast<const T*>(r.a.Wd);
    const int c0 = (int)((int64_t)r.a.chunks * blockIdx.x / r.splits), c1 = (int)((int64_t)r.a.chunks * (blockIdx.x + 1) / r.splits);
    for (int i = t; i < R * D; i += 256) x[i / D][i % D] = i / D < r.a.rows ? widen(static_cast<const T*>(r.a.X)[i]) : 0.f;
    const int m = t & (kHid - 1), kg = t / kHid, o = t % D, hg = t / D;
    float y[R];
#pragma unroll
    for (int i = 0; i < R; ++i) y[i] = 0.f;
    __syncthreads();
    for (int c = c0; c < c1; ++c) {
        const int h = c * kHid + m, hh = min(h, F - 1);
        T wg[K], wu[K], wd[H];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            wg[k] = Wg[(size_t)(kg * K + k) * F + hh];
            wu[k] = Wu[(size_t)(kg * K + k) * F + hh];
        }
#pragma unroll
        for (int k = 0; k < H; ++k) wd[k] = Wd[(size_t)min(c * kHid + hg * H + k, F - 1) * D + o];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float g = 0.f, u = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                g += x[i][kg * K + k] * widen(wg[k]);
                u += x[i][kg * K + k] * widen(wu[k]);
            }
            part[kg][i][0][m] = g;
            part[kg][i][1][m] = u;
        }
        __syncthreads();
        if (t < R * kHid) {
            const int i = t / kHid;
            float g = 0.f, u = 0.f;
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                g += part[k][i][0][m];
                u += part[k][i][1][m];
            }
            hid[i][m] = h < F ? act<ACT>(g) * u : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < H; ++k) {
            const bool ok = c * kHid + hg * H + k < F;           // (a weight past the last hidden value is not one)
#pragma unroll
            for (int i = 0; i < R; ++i) y[i] += ok ? hid[i][hg * H + k] * widen(wd[k]) : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) sums[hg][i][o] = y[i];
    __syncthreads();
    for (int i = t; i < R * D; i += 256) {
        const int row = i / D;
        if (row >= r.a.rows) break;
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < HG; ++k) v += sums[k][row][i % D];
        if (r.splits > 1) r.part[(int64_t)blockIdx.x * r.a.rows * D + i] = v;
        else static_cast<T*>(r.out)[i] = narrow<T>(v);
    }
}

// Workgroups [0, row_blocks * r.splits) form dX, the others the weights' gradients.
template <int D, int PL, int ACT>
__global__ __launch_bounds__(64 * kRowWaves, 1) void ffn_few_bwd_kernel(RowsArgs r, FfnGradArgs k, int row_blocks) {
    extern __shared__ unsigned char lds[];
    const int b = blockIdx.x, n = row_blocks * r.splits;
    if (b < n) {
        few_rows_block<D, PL, ACT, true>(r, b % row_blocks, b / row_blocks, lds);
    } else if (k.splits == 1) {
        grad_block<D, PL, ACT, true>(k, 0, b - n, lds);
    } else {
        grad_block<D, PL, ACT, false>(k, (b - n) % k.splits, (b - n) / k.splits, lds);
    }
}

// Workgroups [0, row_blocks): the shares of the rows; the others: of the weights' gradients.
template <typename T>
__global__ __launch_bounds__(256) void ffn_few_sum_kernel(RowsArgs r, FfnGradArgs k, int D, int row_blocks) {
    __shared__ float lds[16][64];
    const int b = blockIdx.x;
    if (b < row_blocks) combine_block(r.part, r.splits, r.a.rows * D, static_cast<T*>(r.out), r.accumulate, b);
    else grad_reduce_block<T>(k, D, b - row_blocks, lds);
}

// (one or two units of 32 rows need no division)
int few_grad_splits(const rgnn_ffn_desc_t* d) { return d->rows <= 2 * UNIT ? 1 : ffn_grad_shares(d, std::max(1, 256 / ffn_grad_groups(d))); }
// Chunks that stay together; more are divided as long as that puts a workgroup more on each compute unit, among 64 workgroups at most (a lane adds
// all shares of its values).  Forward, that is a second launch, and for bf16, whose chunks are short, three are done sooner; backward the sums'
// launch is there anyway with more than 64 rows, and otherwise costs less than a chunk but for bf16 up to width 64.  In us, undivided / divided:
//   forward   d 64, bf16: 2 chunks, 256 rows 5.6 / 6.5, 3 chunks 7.0 / 7.0; fp32: 2 chunks 9.5 / 9.2 (a call, with its launches, 9.3 / 9.6), 3 chunks 12.0 / 9.5
//   backward  2 chunks, 256 rows, d 32, bf16: 9.2 / 7.4; d 64, fp32: 18.7 / 13.4; d 128, bf16: 20.0 / 14.3
//             60 rows, 2 chunks, d 64, bf16: 9.0 / 10.9; 3 chunks, d 64, bf16: 11.0 / 11.9, fp32: 17.9 / 11.7; d 128, bf16: 18.7 / 13.2
int kept_together(const rgnn_ffn_desc_t* d, bool backward) {
    const bool bf16 = d->dtype == RGNN_BF16;
    return backward ? bf16 && d->width < 128 && few_grad_splits(d) == 1 ? 3 : 1 : bf16 ? 3 : 2;
}
int row_splits(const rgnn_ffn_desc_t* d, bool backward) {
    return ffn_chunks(d) <= kept_together(d, backward) ? 1 : std::max(1, std::min({ffn_chunks(d), 64, 256 / std::max(ffn_row_blocks(d), 1)}));
}
// Rows up to which the forward takes no matrix instructions.  Theirs, of bf16, are as soon done with two rows.  In us, with them / without:
//   1 row          d 64, f 256, bf16: 5.5 / 4.7, fp32: 6.9 / 4.7; d 128, f 341, bf16: 7.3 / 6.2, fp32: 10.2 / 5.8; f 2048, bf16: 10.4 / 9.2, fp32: 13.8 / 9.4
//   2, 3, 4 rows   d 64, f 256, bf16: 5.5 / 5.9, fp32: 7.0 / 5.8; d 128, f 341, bf16: 7.3 / 8.7, fp32: 10.4 / 8.8; f 2048, bf16: 10.4 / 11.9, fp32: 13.5 / 12.1
constexpr int kSingleRows = 4;
bool single(const rgnn_ffn_desc_t* d) { return d->rows <= (d->dtype == RGNN_F32 ? kSingleRows : 1); }
size_t share_bytes(const rgnn_ffn_desc_t* d, bool backward) {
    const int s = row_splits(d, backward);
    return s > 1 ? align_up(sizeof(float) * (size_t)s * d->rows * d->width) : 0;
}
size_t grad_bytes(const rgnn_ffn_desc_t* d) {
    const int s = few_grad_splits(d);
    return s > 1 ? align_up(sizeof(float) * (size_t)s * 3 * d->width * ffn_chunks(d) * kHid) : 0;
}

rgnn_status_t sum(const rgnn_ffn_desc_t* d, const RowsArgs& r, const FfnGradArgs& k, hipStream_t st) {
    const unsigned rows = r.splits > 1 ? (unsigned)((d->rows * d->width / 4 + 255) / 256) : 0;
    const unsigned grads = k.splits > 1 ? (unsigned)((int64_t)3 * d->width * ffn_chunks(d) * kHid / 64) : 0;
    if (rows + grads == 0) return RGNN_OK;
    KernelTimer timer(st, "ffn_few.sum");
    if (d->dtype == RGNN_BF16) ffn_few_sum_kernel<bf16_t><<<rows + grads, 256, 0, st>>>(r, k, d->width, (int)rows);
    else ffn_few_sum_kernel<float><<<rows + grads, 256, 0, st>>>(r, k, d->width, (int)rows);
    RGNN_CHECK_LAUNCH();
    return RGNN_OK;
}

}  // namespace

// Whether this is faster than laying out the weights first.  Every 128 rows read and split all weights again, and a workgroup waits for each of its chunks;
// that is for few rows, or few chunks.
// Forward, chunks that stay together: one launch for two, with as many chunks as take less than the second launch.  Divided ones: the shares to write
// and add grow with the rows, what the laid-out pass takes longer at the least with the chunks and the width: up to sqrt(60 d f) rows (fp32 400), f up to 2048.
// Backward, always a second launch: by rows, types and width, and of width 32, whose chunks are the shortest, fewer rows where there are several of them.
// Microseconds of a call, hidden values f and rows, here / laid out first:
//   forward  d 32, bf16: f 64, 1000: 5.0 / 7.5; 32000: 5.3 / 7.7; f 128, 512: 7.2 / 7.5; 5000: 7.3 / 7.5; f 512, 512: 7.8 / 8.3; 2500: 9.5 / 7.8; 32000: 20.6 / 13.2; f 2048, 1500: 12.8 / 13.4; 5000: 19.4 / 13.5; 32000: 74.0 / 37.4
//   forward  d 32, fp32: f 96, 1000: 8.4 / 8.0; 16000: 11.9 / 8.6; f 512, 1500: 10.2 / 11.4; 5000: 13.7 / 11.7; f 2048, 3500: 23.7 / 26.5; 32000: 121 / 76.7
//   forward  d 64, bf16: f 64, 8000: 6.0 / 7.8; f 256, 512: 7.5 / 7.7; 2500: 9.5 / 7.7; f 2048, 2500: 18.3 / 19.3; 8000: 30.8 / 19.9
//   forward  d 64, fp32: f 64, 1000: 9.6 / 9.0; f 256, 2500: 12.3 / 12.3; 5000: 16.6 / 12.5; f 2048, 5000: 40.7 / 47.5
//   forward  d 128, bf16: f 32, 1000: 6.5 / 7.8; f 64, 1000: 8.4 / 7.8; f 512, 1500: 14.9 / 15.0; 5000: 20.7 / 15.1
//   forward  d 128, fp32: f 32, 1000: 11.5 / 13.3; f 64, 1000: 15.9 / 12.7; f 512, 5000: 31.2 / 38.3; 12000: 50.4 / 39.8
//   backward d 32, bf16: f 32, 16000: 12.6 / 13.6; f 128, 5000: 13.0 / 13.7; 16000: 19.7 / 17.1; f 2048, 8000: 50.3 / 64.2; 16000: 83.1 / 67.6
//   backward d 32, fp32: f 256, 32000: 44.3 / 46.4; f 2048, 12000: 131 / 138; 32000: 289 / 270
//   backward d 64, bf16: f 128, 2500: 14.4 / 15.7; 8000: 25.9 / 19.2; f 2048, 5000: 75.8 / 80.1; 8000: 104 / 83.0
//   backward d 64, fp32: f 256, 8000: 39.2 / 41.6; 12000: 51.8 / 42.8
//   backward d 128, bf16: f 256, 2500: 29.7 / 30.5; 5000: 35.4 / 31.6
//   backward d 128, fp32: f 256, 5000: 60.3 / 67.6; 12000: 93.5 / 77.2
bool ffn_few(const rgnn_ffn_desc_t* d, bool backward) {
    const bool f32 = d->dtype == RGNN_F32;
    const int chunks = ffn_chunks(d);
    if (backward) {
        if (d->width == 32) return d->rows <= (f32 ? chunks <= 8 ? 32768 : 12288 : chunks == 1 ? 32768 : 8192);
        return d->rows <= (f32 ? d->width == 64 ? 8192 : 6144 : d->width == 64 ? 3584 : 2944);
    }
    if (single(d)) return true;
    if (chunks <= kept_together(d, false)) return d->rows <= 32768 && (chunks == 1 || chunks * d->width * (f32 ? 3 : 1) <= 192);
    return d->rows <= 8192 && d->rows * d->rows <= (int64_t)(f32 ? 400 : 60) * d->width * std::min(d->hidden, 2048);
}
size_t ffn_few_bytes(const rgnn_ffn_desc_t* d, bool backward) { return std::max<size_t>(256, share_bytes(d, backward) + (backward ? grad_bytes(d) : 0)); }

rgnn_status_t ffn_few_fwd(const rgnn_ffn_desc_t* d, const FfnArgs& a, void* out, void* workspace, hipStream_t st) {
    const RowsArgs r{a, nullptr, out, static_cast<float*>(workspace), row_splits(d, false), 0};
    auto run = [&]() -> rgnn_status_t {
        RGNN_DISPATCH_FFN(d, {
            if (single(d)) {
                using T = typename std::conditional<PL == 1, bf16_t, float>::type;
                KernelTimer timer(st, "ffn_single_fwd");
                if (PL == 1 || d->rows == 1) ffn_single_fwd_kernel<D, T, ACT, 1><<<r.splits, 256, 0, st>>>(r);
                else if constexpr (PL == 3) ffn_single_fwd_kernel<D, T, ACT, kSingleRows><<<r.splits, 256, 0, st>>>(r);
                RGNN_CHECK_LAUNCH();
                return RGNN_OK;
            }
            constexpr int lds = rows_lds<D, PL, false>();
            auto* const kernel = ffn_few_fwd_kernel<D, PL, ACT>;
            RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds));
            KernelTimer timer(st, "ffn_few_fwd");
            kernel<<<dim3(ffn_row_blocks(d), r.splits), 64 * kRowWaves, lds, st>>>(r);
            RGNN_CHECK_LAUNCH();
            return RGNN_OK;
        });
    };
    RGNN_TRY(run());
    FfnGradArgs k{};
    k.splits = 1;
    return sum(d, r, k, st);
}

rgnn_status_t ffn_few_bwd(const rgnn_ffn_desc_t* d, const FfnArgs& a, void* dX, void* dWg, void* dWu, void* dWd, void* workspace, hipStream_t st) {
    const int accumulate = (d->flags & RGNN_FLAG_ACCUMULATE) != 0;
    RowsArgs r{a, nullptr, dX, static_cast<float*>(workspace), row_splits(d, true), accumulate};
    FfnGradArgs k{a, reinterpret_cast<float*>(static_cast<char*>(workspace) + share_bytes(d, true)), few_grad_splits(d), ffn_grad_groups(d), dWg, dWu, dWd, accumulate};
    const int rows = dX ? ffn_row_blocks(d) : 0, grads = dWg ? k.splits * k.groups : 0;
    if (rows + grads == 0) return RGNN_OK;
    auto run = [&]() -> rgnn_status_t {
        RGNN_DISPATCH_FFN(d, {
            constexpr int lds = std::max(rows_lds<D, PL, true>(), Cut<D, PL>::lds);
            auto* const kernel = ffn_few_bwd_kernel<D, PL, ACT>;
            RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds));
            KernelTimer timer(st, "ffn_few_bwd");
            kernel<<<rows * r.splits + grads, 64 * kRowWaves, lds, st>>>(r, k, rows);
            RGNN_CHECK_LAUNCH();
            return RGNN_OK;
        });
    };
    RGNN_TRY(run());
    if (!rows) r.splits = 1;
    if (!grads) k.splits = 1;
    return sum(d, r, k, st);
}

}  // namespace rgnn
