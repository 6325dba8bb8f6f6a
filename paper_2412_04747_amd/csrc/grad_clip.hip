// Global norm of many gradient tensors, and clipping by it.
//
//   norm = sqrt(sum_t sum_i g_ti^2),  c = min(1, max_norm / (norm + 1e-6)),  clipped = c g
//
// Two reads of every gradient and one write: the memory's rate is the bound, and for a small model the two launches.  Every
// workgroup of the first takes a piece of one tensor and leaves the sum of its squares; every workgroup of the second adds up all those sums
// itself, in the same order (32 KB at most from the L2, less than a launch in between costs), and scales a piece.  A piece is one tensor's, so that
// thousands of small tensors are as many pieces: of more than kDirect sums, a launch in between first adds as many at a time.
// Squares and sums are fp64: 3e38 squared is in range, and a norm over 10^9 terms is right to the last bit of fp32.  That costs nothing: 66M fp32 elements
// clipped into other memory take 150 us, 5.3 TB/s of two reads and a write, what a copy reaches.
// The tensors come as a table in the kernel arguments, so that nothing is copied to the device and a captured call keeps its table.
#include <float.h>
#include <math.h>
#include <algorithm>
#include <vector>

#include "rgnn_internal.h"
#include "device_utils.h"
#include "row_ops.h"

namespace rgnn {

namespace {

constexpr int kThreads = 256;
constexpr int kTable = 128;              // tensors per launch: 3.7 KB of the 4 KB a kernel's arguments may have;
constexpr int kSmallTable = 16;          // of a launch of few, which need not carry them
constexpr int kPieces = 2048;            // about as many pieces in all: eight workgroups per compute unit
constexpr int64_t kMinPiece = 4096;      // elements
constexpr int kDirect = 4096;            // sums that a workgroup adds: 2^24, the most pieces of a call, are 4096 of 4096

template <int N>
struct Table {
    const void* g[N];
    void* out[N];
    int64_t n[N];                    // elements; bit 63: bf16
    int32_t first[N + 1];            // first workgroup of the tensor
    int count;
};
constexpr int64_t kIsBf16 = INT64_MIN;

struct Piece { const void* g; void* out; int64_t beg, end; bool bf16; };

// The workgroup's piece: the last tensor whose first workgroup is not after it.  (Empty tensors have no workgroups.)
template <int N>
__device__ __forceinline__ Piece find_piece(const Table<N>& t, int64_t piece, int block) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= block) lo = mid;
        else hi = mid - 1;
    }
    const int64_t n = t.n[lo] & ~kIsBf16, beg = ((int64_t)block - t.first[lo]) * piece;
    return Piece{t.g[lo], t.out[lo], beg, min(beg + piece, n), t.n[lo] < 0};
}

// Calls fv(i, n) with n vectors of V elements at i, i + kThreads V, .. over [beg, end) where `vec` (four at once, so that four loads are on their way),
// and f1(i) with the single elements left.
template <int V, typename FV, typename F1>
__device__ __forceinline__ void for_piece(int64_t beg, int64_t end, bool vec, FV fv, F1 f1) {
    int64_t i = beg;
    if (vec) {
        constexpr int64_t step = kThreads * V;
        const int64_t whole = beg + (end - beg) / V * V;
        int64_t k = beg + (int64_t)threadIdx.x * V;
        for (; k + 3 * step < whole; k += 4 * step) fv(k, std::integral_constant<int, 4>{});
        for (; k < whole; k += step) fv(k, std::integral_constant<int, 1>{});
        i = whole;
    }
    for (i += threadIdx.x; i < end; i += kThreads) f1(i);
}

// 16-byte vectors need the tensor's address aligned (pieces begin at multiples of 8 elements); a slice that starts elsewhere is
// read element by element, as coalesced.
__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <typename T>
__device__ __forceinline__ double squares(const T* g, int64_t beg, int64_t end) {
    constexpr int V = RowT<T>::V;
    double s[2] = {0.0, 0.0};
    for_piece<V>(beg, end, aligned16(g), [&](int64_t i, auto n) {
        float v[n()][V];
#pragma unroll
        for (int k = 0; k < n(); ++k) load_cols<V>(g + i + k * kThreads * V, v[k]);
#pragma unroll
        for (int k = 0; k < n(); ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) s[e & 1] += (double)v[k][e] * (double)v[k][e];
    }, [&](int64_t i) {
        const double v = widen(g[i]);
        s[0] += v * v;
    });
    return s[0] + s[1];
}

template <int N>
__global__ __launch_bounds__(kThreads) void grad_squares_kernel(Table<N> t, int64_t piece, double* sums) {
    __shared__ double lds[kThreads / 64];
    const Piece p = find_piece(t, piece, blockIdx.x);
    const double s = block_sum(p.bf16 ? squares(static_cast<const bf16_t*>(p.g), p.beg, p.end)
                                      : squares(static_cast<const float*>(p.g), p.beg, p.end), lds);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads) void grad_fold_kernel(const double* sums, int num_sums, double* folded) {
    __shared__ double lds[kThreads / 64];
    const int beg = blockIdx.x * kDirect, end = min(beg + kDirect, num_sums);
    double s = 0.0;
    for (int i = beg + threadIdx.x; i < end; i += kThreads) s += sums[i];
    s = block_sum(s, lds);
    if (threadIdx.x == 0) folded[blockIdx.x] = s;
}

template <typename T>
__device__ __forceinline__ void scale(const T* g, T* out, int64_t beg, int64_t end, float c0, float c) {
    constexpr int V = RowT<T>::V;
    for_piece<V>(beg, end, aligned16(g) && aligned16(out), [&](int64_t i, auto n) {
        float v[n()][V];
#pragma unroll
        for (int k = 0; k < n(); ++k) load_cols<V>(g + i + k * kThreads * V, v[k]);
#pragma unroll
        for (int k = 0; k < n(); ++k) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[k][e] = v[k][e] * c0 * c;
            store_cols<V>(out + i + k * kThreads * V, v[k]);
        }
    }, [&](int64_t i) { out[i] = narrow<T>(widen(g[i]) * c0 * c); });
}

// Workgroup 0 stores the norm (null in the launches after the first).  t.count == 0: the norm alone.
template <int N>
__global__ __launch_bounds__(kThreads) void grad_scale_kernel(Table<N> t, int64_t piece, const double* sums, int num_sums, float max_norm, float* norm) {
    __shared__ double lds[kThreads / 64];
    double s = 0.0;
    for (int i = threadIdx.x; i < num_sums; i += kThreads) s += sums[i];
    const double total = sqrt(block_sum(s, lds));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    if (t.count == 0) return;
    double c = max_norm / (total + 1e-6);
    if (c > 1.0 || (max_norm == INFINITY && total == total)) c = 1.0;      // (a NaN stays one)
    // last pieces first: they are what the caches still hold of the first pass
    const Piece p = find_piece(t, piece, gridDim.x - 1 - blockIdx.x);
    if (c == 1.0 && p.g == p.out) return;
    // (a coefficient below fp32's normal range, of a norm up to 2^21 times the largest value, in two factors)
    const bool low = c > 0.0 && c < FLT_MIN;
    const float c0 = low ? 0x1p-100f : 1.f, c1 = (float)(low ? c * 0x1p100 : c);
    if (p.bf16) scale(static_cast<const bf16_t*>(p.g), static_cast<bf16_t*>(p.out), p.beg, p.end, c0, c1);
    else scale(static_cast<const float*>(p.g), static_cast<float*>(p.out), p.beg, p.end, c0, c1);
}

// Pieces of the tensors: all of one length, a multiple of 8 elements.
struct Plan {
    int64_t piece, pieces, folds;        // folds: sums of kDirect pieces' each, 0 where the pieces' are added directly
    size_t bytes() const { return sizeof(double) * (size_t)(pieces + folds); }
};
rgnn_status_t plan(int64_t count, const int64_t* sizes, Plan* p) {
    if (count < 0) RGNN_FAIL(RGNN_EINVAL, "count %lld is negative", (long long)count);
    if (count > 0 && !sizes) RGNN_FAIL(RGNN_EINVAL, "sizes is NULL");
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] < 0 || sizes[i] > (int64_t)1 << 40) RGNN_FAIL(RGNN_EINVAL, "size %lld of tensor %lld out of range", (long long)sizes[i], (long long)i);
        total += sizes[i];
        if (total > (int64_t)1 << 42) RGNN_FAIL(RGNN_EINVAL, "the tensors have over 2^42 elements");
    }
    p->piece = std::max(kMinPiece, (total / kPieces + 7) / 8 * 8);
    p->pieces = 0;
    for (int64_t i = 0; i < count; ++i) p->pieces += (sizes[i] + p->piece - 1) / p->piece;
    if (p->pieces > 1 << 24) RGNN_FAIL(RGNN_EUNSUPPORTED, "%lld tensors are too many", (long long)count);
    p->folds = p->pieces > kDirect ? (p->pieces + kDirect - 1) / kDirect : 0;
    return RGNN_OK;
}

// Every written range against all others, in order of address.  Reads may share memory among themselves.
rgnn_status_t check_overlaps(int64_t count, const void* const* grads, void* const* clipped, const int64_t* sizes, const int32_t* dtypes, const float* norm,
                             const void* workspace, size_t workspace_bytes) {
    struct R { const char *beg, *end; bool written; int64_t i; };
    std::vector<R> r;
    r.reserve(2 * count + 2);
    auto add = [&](const void* p, size_t n, bool w, int64_t i) { r.push_back({static_cast<const char*>(p), static_cast<const char*>(p) + n, w, i}); };
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] == 0) continue;
        const size_t n = (size_t)sizes[i] * (dtypes[i] == RGNN_BF16 ? 2 : 4);
        if (!clipped || clipped[i] != grads[i]) add(grads[i], n, false, i);
        if (clipped) add(clipped[i], n, true, i);
    }
    add(norm, sizeof(float), true, -1);
    add(workspace, workspace_bytes, true, -2);
    std::sort(r.begin(), r.end(), [](const R& a, const R& b) { return a.beg < b.beg; });
    const char* any_end = nullptr;           // end of what began before, and of what is written of it
    const char* written_end = nullptr;
    for (const R& x : r) {
        if (x.beg < (x.written ? any_end : written_end))
            RGNN_FAIL(RGNN_EINVAL, "%s overlaps another tensor", x.i == -1 ? "norm" : x.i == -2 ? "the workspace" : x.written ? "a clipped tensor" : "a gradient");
        any_end = std::max(any_end, x.end);
        if (x.written) written_end = std::max(written_end, x.end);
    }
    return RGNN_OK;
}

}  // namespace

}  // namespace rgnn

using namespace rgnn;

extern "C" rgnn_status_t rgnn_clip_workspace_bytes(int64_t count, const int64_t* sizes, size_t* workspace) {
    Plan p;
    RGNN_TRY(plan(count, sizes, &p));
    if (!workspace) RGNN_FAIL(RGNN_EINVAL, "workspace is NULL");
    *workspace = align_up(std::max(p.bytes(), sizeof(double)));
    return RGNN_OK;
}

extern "C" rgnn_status_t rgnn_clip_grad_norm(int64_t count, const void* const* grads, void* const* clipped, const int64_t* sizes,
                                             const int32_t* dtypes, float max_norm, float* norm, void* workspace, void* stream) {
    Plan p;
    RGNN_TRY(plan(count, sizes, &p));
    if (count > 0 && (!grads || !dtypes)) RGNN_FAIL(RGNN_EINVAL, "grads or dtypes is NULL");
    if (!norm) RGNN_FAIL(RGNN_EINVAL, "norm is NULL");
    if (clipped && !(max_norm >= 0.f)) RGNN_FAIL(RGNN_EINVAL, "max_norm is not a number >= 0");
    if (!workspace) RGNN_FAIL(RGNN_EWORKSPACE, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(workspace) % 16 || reinterpret_cast<uintptr_t>(norm) % 4) RGNN_FAIL(RGNN_EINVAL, "workspace or norm is not aligned");
    for (int64_t i = 0; i < count; ++i) {
        RGNN_TRY(check_dtype(dtypes[i]));
        if (sizes[i] == 0) continue;
        if (!grads[i] || (clipped && !clipped[i])) RGNN_FAIL(RGNN_EINVAL, "tensor %lld is NULL", (long long)i);
        const uintptr_t at = reinterpret_cast<uintptr_t>(grads[i]) | (clipped ? reinterpret_cast<uintptr_t>(clipped[i]) : 0);
        if (at % (dtypes[i] == RGNN_BF16 ? 2 : 4)) RGNN_FAIL(RGNN_EINVAL, "tensor %lld is not aligned to its elements", (long long)i);
    }
    try {
        RGNN_TRY(check_overlaps(count, grads, clipped, sizes, dtypes, norm, workspace, p.bytes()));
    } catch (const std::bad_alloc&) {
        RGNN_FAIL(RGNN_ENOMEM, "out of host memory");
    }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    double* const sums = static_cast<double*>(workspace);
    // launches of up to kTable tensors that have elements; `f` gets the table and its number of workgroups
    auto tables = [&](auto f) -> rgnn_status_t {
        Table<kTable> t;
        t.count = 0;
        t.first[0] = 0;
        for (int64_t i = 0; i < count; ++i) {
            if (sizes[i] > 0) {
                const int k = t.count++;
                t.g[k] = grads[i];
                t.out[k] = clipped ? clipped[i] : nullptr;
                t.n[k] = sizes[i] | (dtypes[i] == RGNN_BF16 ? kIsBf16 : 0);
                t.first[k + 1] = t.first[k] + (int32_t)((sizes[i] + p.piece - 1) / p.piece);
            }
            if (t.count == kTable || (i + 1 == count && t.count > 0)) {
                RGNN_TRY(f(t, t.first[t.count]));
                t.count = 0;
            }
        }
        return RGNN_OK;
    };
    int64_t at = 0;
    auto fitting = [](const Table<kTable>& t, auto f) {
        if (t.count > kSmallTable) return f(t);
        Table<kSmallTable> s;
        s.count = t.count;
        std::copy(t.g, t.g + t.count, s.g);
        std::copy(t.out, t.out + t.count, s.out);
        std::copy(t.n, t.n + t.count, s.n);
        std::copy(t.first, t.first + t.count + 1, s.first);
        return f(s);
    };
    RGNN_TRY(tables([&](const Table<kTable>& t, int blocks) -> rgnn_status_t {
        KernelTimer timer(st, "grad_squares");
        fitting(t, [&](const auto& u) { grad_squares_kernel<<<blocks, kThreads, 0, st>>>(u, p.piece, sums + at); });
        RGNN_CHECK_LAUNCH();
        at += blocks;
        return RGNN_OK;
    }));
    const double* added = sums;
    int num_added = (int)p.pieces;
    if (p.folds) {
        KernelTimer timer(st, "grad_fold");
        grad_fold_kernel<<<(unsigned)p.folds, kThreads, 0, st>>>(sums, (int)p.pieces, sums + p.pieces);
        RGNN_CHECK_LAUNCH();
        added = sums + p.pieces;
        num_added = (int)p.folds;
    }
    bool stored = false;
    auto scale_launch = [&](const Table<kTable>& t, int blocks) -> rgnn_status_t {
        KernelTimer timer(st, "grad_scale");
        fitting(t, [&](const auto& u) { grad_scale_kernel<<<blocks, kThreads, 0, st>>>(u, p.piece, added, num_added, max_norm, stored ? nullptr : norm); });
        RGNN_CHECK_LAUNCH();
        stored = true;
        return RGNN_OK;
    };
    if (clipped) RGNN_TRY(tables(scale_launch));
    if (!stored) {
        Table<kTable> none;
        none.count = 0;
        none.first[0] = 0;
        RGNN_TRY(scale_launch(none, 1));
    }
    return RGNN_OK;
}
