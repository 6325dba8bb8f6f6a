// Residual addition with root-mean-square norm, forward and backward.
//
//   s = x + r,  q = 1 / sqrt(mean(s^2) + eps),  out = s q w
// With g = dOut w, the derivative of out_j = s_j q w_j is q (delta_ij - s_i s_j q^2 / d), so
//   dS = dSum + q (g - s q^2 mean(g s)),   dw = sum over the rows of dOut s q.
//
// Ten operations per element against 8 to 16 bytes: the memory's rate is the bound.  A row stays in the registers of the lanes
// that loaded it (16 bytes each where the width allows), so each tensor is passed once; the two means of the backward are summed
// over those lanes together, and q is formed again from s instead of being stored.  Narrow rows share a wavefront: a row of 64
// fp32 columns is 16 lanes.  Rows of more than 256 vectors are a workgroup's.
// Measured against 4.8 .. 5.3 TB/s of a large copy: 1M rows of 64, fp32 to bf16, forward 181 us (4.9 TB/s); 2M rows of 128, bf16, forward 380 us (5.4),
// backward 430 (4.8).
// The sum of squares is fp32.  A row whose squares leave its range, values past 1e17 at width 8192 or 1e19 alone, is summed again with its values scaled
// down by a power of two; s is in registers, so that the other rows pay a comparison and a multiplication by one.
// dw: a workgroup walks its rows with its columns' sums in registers and leaves one partial row; a second launch sums those in order,
// so results do not depend on timing.
#include <float.h>

#include "rgnn_internal.h"
#include "device_utils.h"
#include "row_ops.h"

namespace rgnn {

namespace {

constexpr int kBlock = 512;              // threads of a workgroup
// Four workgroups per compute unit hold all 32 wavefronts of its SIMDs, where the registers allow it: the forward of up to 16 columns per lane.  The backward
// takes 88 to 98 registers with two vectors of four (two resident), 76 with one of eight (three): its workgroups then come in uneven turns.
constexpr int kMaxBlocks = 1024;
constexpr int kMaxWidth = 8192;

// Columns c .. c + V - 1 of a row, those before `width`.  EVEN: the width is a multiple of V and rows start at multiples of 16 bytes (8 for
// four bf16); otherwise the last vector may be short, and vectors lie at any multiple of their element's size, which the
// hardware loads and stores as well (with single columns / so: 2M rows of 33 fp32 columns, backward, 318 / 205 us; 100000 rows of 257 bf16
// columns, forward, 123 / 45; 30011 rows of 349 fp32 columns, backward, 44 / 35).
template <bool EVEN, int V, typename T>
__device__ __forceinline__ void load_v(const T* row, int c, int width, float (&v)[V]) {
    if constexpr (EVEN) {
        load_cols<V>(row + c, v);
    } else if (c + V <= width) {
        T t[V];
        __builtin_memcpy(t, row + c, sizeof(t));
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = widen(t[e]);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = c + e < width ? widen(row[c + e]) : 0.f;
    }
}
template <bool EVEN, int V, typename T>
__device__ __forceinline__ void store_v(T* row, int c, int width, const float (&v)[V]) {
    if constexpr (EVEN) {
        store_cols<V>(row + c, v);
    } else if (c + V <= width) {
        T t[V];
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] = narrow<T>(v[e]);
        __builtin_memcpy(row + c, t, sizeof(t));
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < width) row[c + e] = narrow<T>(v[e]);
    }
}

// Sum over the G lanes of a row (G a power of two up to 64), or over the workgroup.
__device__ __forceinline__ float lanes_sum(float v, int G) {
    if (G >= 2) v += dpp_move<kDppQuadSwap1>(v);
    if (G >= 4) v += dpp_move<kDppQuadSwap2>(v);
    if (G >= 8) v += dpp_move<kDppHalfMirror>(v);
    if (G >= 16) v += dpp_move<kDppMirror>(v);
    if (G >= 32) v += __shfl_xor(v, 16);
    if (G >= 64) v += __shfl_xor(v, 32);
    return v;
}

// How a workgroup's lanes share rows: G lanes per row (kBlock: the whole workgroup).
struct Shape {
    int G, rows_per_block, lane, group;
    __device__ __forceinline__ explicit Shape(int g) : G(g), rows_per_block(kBlock / g), lane(threadIdx.x & (g - 1)), group(threadIdx.x / g) {}
};

// Two sums over the lanes of a row.  `lds` holds two floats per wavefront, twice (rows in turn use either half, so that one barrier
// per row is enough).
__device__ __forceinline__ void row_sums(float& a, float& b, int G, float* lds, int turn) {
    a = lanes_sum(a, min(G, 64));
    b = lanes_sum(b, min(G, 64));
    if (G <= 64) return;
    constexpr int W = kBlock / 64;
    float* const at = lds + (turn & 1) * 2 * W;
    if ((threadIdx.x & 63) == 0) {
        at[threadIdx.x >> 6] = a;
        at[W + (threadIdx.x >> 6)] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        a += at[i];
        b += at[W + i];
    }
}

// What a row's values are multiplied by where their squares' sum is infinite.  Any finite row's sum is in range then, 2^-32 or more, and the squares
// that vanish are below 2^-149.
constexpr float kScaleDown = 0x1p-80f;

struct FwdArgs {
    int64_t rows;
    int width, G;
    float eps;
    const void* x; const void* r; const float* w;
    void* sum; void* out;
};

// (Two vectors of eight columns: 63 registers and eight wavefronts per SIMD; the compiler would take 66 and seven, three workgroups instead of four.
// 100000 rows of 1024 bf16 columns: 148 us, 169 with three.)
template <typename TX, typename TS, typename TO, int V, int NV, bool EVEN>
__global__ __launch_bounds__(kBlock, V == 8 && NV == 2 ? 8 : 1) void norm_fwd_kernel(FwdArgs a) {
    __shared__ float lds[4 * (kBlock / 64)];
    const Shape sh(a.G);
    const float inv = 1.f / (float)a.width;
    float w[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (sh.lane + j * sh.G) * V;
        zero_cols<V>(w[j]);
        if (c < a.width) load_v<EVEN>(a.w, c, a.width, w[j]);
    }
    int turn = 0;
    // (the trip count is the same for all threads of a workgroup whose rows are its own: the barrier in row_sums)
    for (int64_t row0 = (int64_t)blockIdx.x * sh.rows_per_block; row0 < a.rows; row0 += (int64_t)gridDim.x * sh.rows_per_block, ++turn) {
        const int64_t row = row0 + sh.group;
        const bool live = row < a.rows;
        const int64_t base = row * a.width;
        float s[NV][V], sq = 0.f, none = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (sh.lane + j * sh.G) * V;
            zero_cols<V>(s[j]);
            if (live && c < a.width) {
                load_v<EVEN>(static_cast<const TX*>(a.x) + base, c, a.width, s[j]);
                if (a.r) {
                    float r[V];
                    load_v<EVEN>(static_cast<const TS*>(a.r) + base, c, a.width, r);
#pragma unroll
                    for (int e = 0; e < V; ++e) s[j][e] += r[e];
                }
            }
            sq += dot_cols<V>(s[j], s[j]);
        }
        row_sums(sq, none, sh.G, lds, turn);
        float k = 1.f;
        if (!(sq <= FLT_MAX)) {              // (all lanes of the row, and where the row is a workgroup's, all of it)
            k = kScaleDown;
            sq = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) sq += (s[j][e] * k) * (s[j][e] * k);
            row_sums(sq, none, sh.G, lds, ++turn);
        }
        // (With a constant on either way the compiler writes all that follows twice.  Of two vectors of eight columns that takes 78 registers instead of 63; of
        // uneven rows it is the faster: 100000 of 257 bf16 columns 43 us, 66 with one copy.)
        if constexpr (EVEN) asm("" : "+v"(k));
        const float q = rsqrtf(sq * inv + a.eps * k * k);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (sh.lane + j * sh.G) * V;
            if (live && c < a.width) {
                if (a.sum) store_v<EVEN>(static_cast<TS*>(a.sum) + base, c, a.width, s[j]);
                float y[V];
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] = s[j][e] * q * k * w[j][e];
                store_v<EVEN>(static_cast<TO*>(a.out) + base, c, a.width, y);
            }
        }
    }
}

struct BwdArgs {
    int64_t rows;
    int width, G, accumulate;
    float eps;
    const void* s; const float* w; const void* dy; const void* ds;
    void* dx; void* dr;
    float* part;             // [gridDim.x][width] or, of a single workgroup, dw itself; null: dw is not wanted
};

template <bool EVEN, typename T, int V>
__device__ __forceinline__ void put(T* row, int c, int width, const float (&v)[V], int accumulate) {
    float t[V];
    zero_cols<V>(t);
    if (accumulate) load_v<EVEN>(row, c, width, t);
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] += v[e];
    store_v<EVEN>(row, c, width, t);
}

template <typename TX, typename TS, typename TO, int V, int NV, bool EVEN>
__global__ __launch_bounds__(kBlock) void norm_bwd_kernel(BwdArgs a) {
    extern __shared__ float lds[];           // row_sums' halves, then a row of sums per wavefront
    const Shape sh(a.G);
    const float inv = 1.f / (float)a.width;
    float w[NV][V], dw[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (sh.lane + j * sh.G) * V;
        zero_cols<V>(w[j]);
        zero_cols<V>(dw[j]);
        if (c < a.width) load_v<EVEN>(a.w, c, a.width, w[j]);
    }
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * sh.rows_per_block; row0 < a.rows; row0 += (int64_t)gridDim.x * sh.rows_per_block, ++turn) {
        const int64_t row = row0 + sh.group;
        const bool live = row < a.rows;
        const int64_t base = row * a.width;
        float s[NV][V], dy[NV][V], ds[NV][V], sq = 0.f, gs = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (sh.lane + j * sh.G) * V;
            zero_cols<V>(s[j]);
            zero_cols<V>(dy[j]);
            zero_cols<V>(ds[j]);
            if (live && c < a.width) {
                load_v<EVEN>(static_cast<const TS*>(a.s) + base, c, a.width, s[j]);
                load_v<EVEN>(static_cast<const TO*>(a.dy) + base, c, a.width, dy[j]);
                if (a.ds) load_v<EVEN>(static_cast<const TS*>(a.ds) + base, c, a.width, ds[j]);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sq += s[j][e] * s[j][e];
                gs += dy[j][e] * w[j][e] * s[j][e];
            }
        }
        row_sums(sq, gs, sh.G, lds, turn);
        float k = 1.f;
        if (!(sq <= FLT_MAX)) {              // as in the forward; the scaled values take their place
            k = kScaleDown;
            sq = gs = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    s[j][e] *= k;
                    sq += s[j][e] * s[j][e];
                    gs += dy[j][e] * w[j][e] * s[j][e];
                }
            row_sums(sq, gs, sh.G, lds, ++turn);
        }
        // (with t = k s: q(s) = k q(t), s q(s)^2 mean(g s) = t q(t)^2 mean(g t))
        const float q = rsqrtf(sq * inv + a.eps * k * k), along = q * q * (gs * inv), qs = q * k;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (sh.lane + j * sh.G) * V;
            if (live && c < a.width) {
                float d[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    d[e] = ds[j][e] + qs * (dy[j][e] * w[j][e] - s[j][e] * along);
                    dw[j][e] += dy[j][e] * (s[j][e] * q);
                }
                if (a.dx) put<EVEN>(static_cast<TX*>(a.dx) + base, c, a.width, d, a.accumulate);
                if (a.dr) put<EVEN>(static_cast<TS*>(a.dr) + base, c, a.width, d, a.accumulate);
            }
        }
    }
    if (!a.part) return;
    float* const mine = a.part + (int64_t)blockIdx.x * a.width;
    const int add = a.accumulate && gridDim.x == 1;
    if (sh.G > 64) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (sh.lane + j * sh.G) * V;
            if (c < a.width) put<EVEN>(mine, c, a.width, dw[j], add);
        }
        return;
    }
    // the rows of a wavefront, then the wavefronts of the workgroup
    float* const per_wave = lds + 4 * (kBlock / 64);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (sh.lane + j * sh.G) * V;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float v = dw[j][e];
            for (int o = sh.G; o < 64; o <<= 1) v += __shfl_xor(v, o);
            if ((threadIdx.x & 63) < sh.G && c + e < a.width) per_wave[(threadIdx.x >> 6) * a.width + c + e] = v;
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += kBlock) {
        float v = 0.f;
        for (int k = 0; k < kBlock / 64; ++k) v += per_wave[k * a.width + c];
        mine[c] = add ? v + mine[c] : v;
    }
}

// dw[c] = sum of the partial rows' column c: 16 columns per workgroup, 64 lanes of rows each.
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float* part, int n, int width, float* dw, int accumulate) {
    __shared__ float lds[64][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), k = threadIdx.x >> 4;
    float v = 0.f;
    if (c < width)
        for (int i = k; i < n; i += 64) v += part[(int64_t)i * width + c];
    lds[k][threadIdx.x & 15] = v;
    __syncthreads();
    for (int h = 32; h > 0; h >>= 1) {
        if (k < h) lds[k][threadIdx.x & 15] += lds[k + h][threadIdx.x & 15];
        __syncthreads();
    }
    if (k == 0 && c < width) dw[c] = lds[0][threadIdx.x & 15] + (accumulate ? dw[c] : 0.f);
}

// Columns per vector, lanes per row and vectors per lane.  A vector is 16 bytes of the narrowest type among the tensors, at most 8
// columns, where the width is a multiple of it; otherwise four columns.  Up to four vectors per lane a row is a wavefront's, whose lanes sum
// without a barrier; a wider one is a workgroup's (8192 columns are four vectors of four again, two of eight).
struct Plan { int V, G, NV, blocks; };
Plan plan(const rgnn_norm_desc_t* d) {
    const bool all16 = d->x_dtype == RGNN_BF16 && d->sum_dtype == RGNN_BF16 && d->out_dtype == RGNN_BF16;
    Plan p;
    p.V = all16 && d->width % 8 == 0 ? 8 : 4;
    const int vectors = (d->width + p.V - 1) / p.V;
    p.G = 1;
    while (p.G < vectors && p.G < 64) p.G *= 2;
    if (vectors > 4 * 64) p.G = kBlock;
    p.NV = (vectors + p.G - 1) / p.G;
    // (what two turns of a workgroup finish is left to one: the backward then needs no second launch)
    const int64_t turns = (d->rows + kBlock / p.G - 1) / (kBlock / p.G);
    p.blocks = turns <= 2 ? (int)std::min<int64_t>(turns, 1) : (int)std::min<int64_t>(kMaxBlocks, turns);
    return p;
}

template <int N> using Int = std::integral_constant<int, N>;
// ALL16: every tensor is bf16
template <bool ALL16, typename F>
rgnn_status_t with_vectors(const rgnn_norm_desc_t* d, const Plan& p, F f) {
    auto count = [&](auto V, auto even) {
        return p.NV <= 1 ? f(V, Int<1>{}, even) : p.NV <= 2 ? f(V, Int<2>{}, even) : f(V, Int<4>{}, even);
    };
    if constexpr (ALL16)
        if (p.V == 8) return count(Int<8>{}, std::true_type{});
    return d->width % 4 == 0 ? count(Int<4>{}, std::true_type{}) : count(Int<4>{}, std::false_type{});
}

template <typename TX, typename TS, typename TO>
rgnn_status_t launch_fwd(const rgnn_norm_desc_t* d, const Plan& p, const FwdArgs& a, hipStream_t st) {
    return with_vectors<sizeof(TX) + sizeof(TS) + sizeof(TO) == 6>(d, p, [&](auto V, auto NV, auto even) -> rgnn_status_t {
        KernelTimer timer(st, "norm_fwd");
        norm_fwd_kernel<TX, TS, TO, V(), NV(), even()><<<p.blocks, kBlock, 0, st>>>(a);
        RGNN_CHECK_LAUNCH();
        return RGNN_OK;
    });
}
template <typename TX, typename TS, typename TO>
rgnn_status_t launch_bwd(const rgnn_norm_desc_t* d, const Plan& p, const BwdArgs& a, hipStream_t st) {
    return with_vectors<sizeof(TX) + sizeof(TS) + sizeof(TO) == 6>(d, p, [&](auto V, auto NV, auto even) -> rgnn_status_t {
        // at most 8 wavefronts' rows of 64 x 4 vectors of eight columns: 64 KB
        const size_t lds = sizeof(float) * (4 + (p.G <= 64 && a.part ? a.width : 0)) * (kBlock / 64);
        RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(norm_bwd_kernel<TX, TS, TO, V(), NV(), even()>), lds));
        KernelTimer timer(st, "norm_bwd");
        norm_bwd_kernel<TX, TS, TO, V(), NV(), even()><<<p.blocks, kBlock, lds, st>>>(a);
        RGNN_CHECK_LAUNCH();
        return RGNN_OK;
    });
}
template <typename F>
rgnn_status_t with_types(const rgnn_norm_desc_t* d, F f) {
    const float f32 = 0;
    const bf16_t b16 = 0;
    auto third = [&](auto x, auto s) { return d->out_dtype == RGNN_BF16 ? f(x, s, b16) : f(x, s, f32); };
    auto second = [&](auto x) { return d->sum_dtype == RGNN_BF16 ? third(x, b16) : third(x, f32); };
    return d->x_dtype == RGNN_BF16 ? second(b16) : second(f32);
}

rgnn_status_t check_desc(const rgnn_norm_desc_t* d) {
    if (!d) RGNN_FAIL(RGNN_EINVAL, "desc is NULL");
    RGNN_TRY(check_rows(d->rows));
    if (d->width < 1) RGNN_FAIL(RGNN_EINVAL, "width %d is not positive", d->width);
    if (d->width > kMaxWidth) RGNN_FAIL(RGNN_EUNSUPPORTED, "width %d not supported (up to %d)", d->width, kMaxWidth);
    for (int32_t t : {d->x_dtype, d->sum_dtype, d->out_dtype}) RGNN_TRY(check_dtype(t));
    if (!(d->eps >= 0.f) || d->eps == INFINITY) RGNN_FAIL(RGNN_EINVAL, "eps is not a finite number >= 0");
    if (d->flags & ~RGNN_FLAG_ACCUMULATE) RGNN_FAIL(RGNN_EINVAL, "flags: only RGNN_FLAG_ACCUMULATE applies");
    return RGNN_OK;
}

}  // namespace

}  // namespace rgnn

using namespace rgnn;

extern "C" rgnn_status_t rgnn_norm_workspace_bytes(const rgnn_norm_desc_t* desc, size_t* bwd_workspace) {
    RGNN_TRY(check_desc(desc));
    if (!bwd_workspace) RGNN_FAIL(RGNN_EINVAL, "bwd_workspace is NULL");
    *bwd_workspace = align_up(sizeof(float) * (size_t)std::max(plan(desc).blocks, 1) * desc->width);
    return RGNN_OK;
}

extern "C" rgnn_status_t rgnn_norm_fwd(const rgnn_norm_desc_t* desc, const void* x, const void* residual, const float* weight, void* sum,
                                       void* out, void* stream) {
    RGNN_TRY(check_desc(desc));
    if (!weight) RGNN_FAIL(RGNN_EINVAL, "weight is NULL");
    if (desc->rows == 0) return RGNN_OK;
    if (!x || !out) RGNN_FAIL(RGNN_EINVAL, "x or out is NULL");
    const size_t n = (size_t)desc->rows * desc->width;
    const Span xs = span(x, n, desc->x_dtype), rs = span(residual, n, desc->sum_dtype), ss = span(sum, n, desc->sum_dtype),
               os = span(out, n, desc->out_dtype), ws = span(weight, desc->width, RGNN_F32);
    for (const Span& s : {xs, rs, ss, os, ws}) RGNN_TRY(check_aligned(s));
    // a row's lanes have read it before they write it: in place is fine, a shifted overlap is not
    for (const Span& o : {ss, os})
        if (o.overlaps(ws) || (o.overlaps(xs) && !o.same(xs)) || (o.overlaps(rs) && !o.same(rs)))
            RGNN_FAIL(RGNN_EINVAL, "sum or out overlaps an input that it is not the buffer of");
    if (ss.overlaps(os)) RGNN_FAIL(RGNN_EINVAL, "sum and out overlap");
    const Plan p = plan(desc);
    const FwdArgs a{desc->rows, desc->width, p.G, desc->eps, x, residual, weight, sum, out};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return with_types(desc, [&](auto tx, auto ts, auto to) { return launch_fwd<decltype(tx), decltype(ts), decltype(to)>(desc, p, a, st); });
}

extern "C" rgnn_status_t rgnn_norm_bwd(const rgnn_norm_desc_t* desc, const void* sum, const float* weight, const void* dOut, const void* dSum,
                                       void* dX, void* dResidual, float* dWeight, void* workspace, void* stream) {
    RGNN_TRY(check_desc(desc));
    if (!weight) RGNN_FAIL(RGNN_EINVAL, "weight is NULL");
    if (dWeight && !workspace) RGNN_FAIL(RGNN_EWORKSPACE, "workspace is NULL");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int accumulate = (desc->flags & RGNN_FLAG_ACCUMULATE) != 0;
    const Plan p = plan(desc);
    RGNN_TRY(check_aligned(span(weight, desc->width, RGNN_F32)));
    RGNN_TRY(check_aligned(span(dWeight, desc->width, RGNN_F32)));
    RGNN_TRY(check_aligned(span(workspace, 1, RGNN_F32)));
    if (desc->rows > 0) {
        if (!sum || !dOut) RGNN_FAIL(RGNN_EINVAL, "sum or dOut is NULL");
        const size_t n = (size_t)desc->rows * desc->width;
        const Span ss = span(sum, n, desc->sum_dtype), ys = span(dOut, n, desc->out_dtype), gs = span(dSum, n, desc->sum_dtype),
                   xs = span(dX, n, desc->x_dtype), rs = span(dResidual, n, desc->sum_dtype), ws = span(weight, desc->width, RGNN_F32),
                   dw = span(dWeight, desc->width, RGNN_F32), wk = span(workspace, dWeight ? (size_t)p.blocks * desc->width : 0, RGNN_F32);
        for (const Span& s : {ss, ys, gs, xs, rs}) RGNN_TRY(check_aligned(s));
        for (const Span& o : {xs, rs})
            if (o.overlaps(ss) || o.overlaps(ws) || o.overlaps(dw) || o.overlaps(wk) || (o.overlaps(ys) && !o.same(ys)) || (o.overlaps(gs) && !o.same(gs)))
                RGNN_FAIL(RGNN_EINVAL, "dX or dResidual overlaps a tensor that it is not the buffer of");
        if (xs.overlaps(rs)) RGNN_FAIL(RGNN_EINVAL, "dX and dResidual overlap");
        for (const Span& o : {dw, wk})
            if (o.overlaps(ss) || o.overlaps(ws) || o.overlaps(ys) || o.overlaps(gs))
                RGNN_FAIL(RGNN_EINVAL, "dWeight or the workspace overlaps an input");
        if (dw.overlaps(wk)) RGNN_FAIL(RGNN_EINVAL, "dWeight and the workspace overlap");
        if (dX || dResidual || dWeight) {
            const BwdArgs a{desc->rows, desc->width, p.G, accumulate, desc->eps, sum, weight, dOut, dSum, dX, dResidual,
                            dWeight ? p.blocks == 1 ? dWeight : static_cast<float*>(workspace) : nullptr};
            RGNN_TRY(with_types(desc, [&](auto tx, auto ts, auto to) { return launch_bwd<decltype(tx), decltype(ts), decltype(to)>(desc, p, a, st); }));
        }
    }
    if (dWeight && p.blocks != 1 && (desc->rows > 0 || !accumulate)) {
        KernelTimer timer(st, "norm_bwd.reduce");
        norm_dw_kernel<<<(desc->width + 15) / 16, 1024, 0, st>>>(static_cast<const float*>(workspace), p.blocks, desc->width, dWeight, accumulate);
        RGNN_CHECK_LAUNCH();
    }
    return RGNN_OK;
}
