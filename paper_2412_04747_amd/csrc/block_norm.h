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
    int streaming;           // sum and out are more than the caches hold
    float eps;
    BlockParams p;
    const void* a; const void* s;
    void* sum; void* out;
    int8_t* a_codes; uint8_t* a_scales; int8_t* s_codes; uint8_t* s_scales;
};

struct BlockBwdArgs {
    int64_t rows;
    int width, G, accumulate;
    int streaming;           // dA and dS are more than the caches hold, and nothing is added to them
    float eps;
    BlockParams p;
    const void* a; const void* s;        // codes, where they are held in 8 bits
    const uint8_t* a_scales; const uint8_t* s_scales;
    const void* dy; const void* ds;
    void* da; void* dstream;
    int sums;                // whether a parameter's gradient is wanted
    float* part;             // by groups of columns, [gridDim.x][T + 1] each: G and dscale of each type, then dw2 (a single workgroup writes the gradients itself)
    rgnn_block_norm_grads_t grads;
};

// Threads of a workgroup: of one that has whole rows to itself, and of one whose wavefronts have them.
constexpr int kNarrowBlock = 256;
__host__ __device__ constexpr int block_threads(int G) { return G == kBlock ? kBlock : kNarrowBlock; }

// Columns per vector, lanes per row (a workgroup's: kBlock) and vectors per lane: as for the norm, but at most 16 columns per lane.
struct JunctionPlan { int V, G, NV; int64_t turns; };
inline JunctionPlan block_plan(const rgnn_block_norm_desc_t* d) {
    const bool all16 = d->a_dtype == RGNN_BF16 && d->sum_dtype == RGNN_BF16 && d->out_dtype == RGNN_BF16;
    JunctionPlan p;
    p.V = all16 && d->width % 8 == 0 && d->width <= 1024 ? 8 : 4;
    const int vectors = (d->width + p.V - 1) / p.V;
    p.G = 1;
    while (p.G < vectors && p.G < 64) p.G *= 2;
    if (vectors > 64 * 16 / p.V) p.G = kBlock;
    p.NV = (vectors + p.G - 1) / p.G;
    const int rows = block_threads(p.G) / p.G;
    p.turns = (d->rows + rows - 1) / rows;
    return p;
}

// Types whose sums a backward's workgroup can hold in the LDS at once: four places of each, or one where a row is a workgroup's (block_norm_bwd.h).  The first bound leaves two
// workgroups of narrow rows to a compute unit; within the second, up to 154 KB, there may be one.  (Backward, fp32, with 1, 3 and 8 types in order: 50000 rows of 1024 in 214, 219 and
// 244 us; with 3 and 8 mixed 225 and 249; 100000 rows of 512 with 4, 7 and 8 types 224, 217 and 232.)
inline bool block_types_fit(int64_t types, int64_t width) {
    return types == 1 || types * (width + 12) <= 4096 || (types <= 32 && width <= 1024 && (types + 1) * (width + 12) <= 9600);
}

// How vectors lie in a row: its width is a multiple of them; or the last one is short; or there is only that.
enum Lie { kUneven, kEven, kNarrow };

// What a kernel's rows look like, as compile-time values: V columns per vector, NV vectors per lane, GC lanes per row (kBlock: all of a workgroup; 0: any number up to 64).
template <int V_, int NV_, int LIE_, int GC_>
struct RowShape { static constexpr int V = V_, NV = NV_, LIE = LIE_, GC = GC_; };

// f(RowShape).  Rows of the layers' widths, 32, 64 and 128, get a kernel for their number of lanes:
// the sums over a row are then without branches.
template <bool ALL16, typename F>
rgnn_status_t block_with_shape(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, F f) {
    if constexpr (ALL16)
        if (p.V == 8) {
            if (d->width == 32) return f(RowShape<8, 1, kEven, 4>{});
            if (d->width == 64) return f(RowShape<8, 1, kEven, 8>{});
            if (d->width == 128) return f(RowShape<8, 1, kEven, 16>{});
            return p.NV <= 1 ? f(RowShape<8, 1, kEven, 0>{}) : f(RowShape<8, 2, kEven, 0>{});
        }
    if (d->width == 32) return f(RowShape<4, 1, kEven, 8>{});
    if (d->width == 64) return f(RowShape<4, 1, kEven, 16>{});
    if (d->width == 128) return f(RowShape<4, 1, kEven, 32>{});
    if (d->width < 4) return f(RowShape<4, 1, kNarrow, 1>{});
    auto lies = [&](auto lie) {
        constexpr int L = decltype(lie)::value;
        if (p.G == kBlock) return p.NV <= 2 ? f(RowShape<4, 2, L, kBlock>{}) : f(RowShape<4, 4, L, kBlock>{});
        return p.NV <= 1 ? f(RowShape<4, 1, L, 0>{}) : p.NV <= 2 ? f(RowShape<4, 2, L, 0>{}) : f(RowShape<4, 4, L, 0>{});
    };
    return d->width % 4 == 0 ? lies(std::integral_constant<int, kEven>{}) : lies(std::integral_constant<int, kUneven>{});
}
template <typename F>
rgnn_status_t block_with_types(const rgnn_block_norm_desc_t* d, F f) {
    const float f32 = 0;
    const bf16_t b16 = 0;
    auto third = [&](auto x, auto s) { return d->out_dtype == RGNN_BF16 ? f(x, s, b16) : f(x, s, f32); };
    auto second = [&](auto x) { return d->sum_dtype == RGNN_BF16 ? third(x, b16) : third(x, f32); };
    return d->a_dtype == RGNN_BF16 ? second(b16) : second(f32);
}

// N words at an address that is a multiple of A.
template <int N, int A> struct Words;
template <> struct Words<1, 1> { typedef unsigned type __attribute__((aligned(1))); };
template <> struct Words<1, 4> { typedef unsigned type; };
template <> struct Words<2, 2> { typedef unsigned type __attribute__((ext_vector_type(2), aligned(2))); };
template <> struct Words<2, 8> { typedef unsigned type __attribute__((ext_vector_type(2))); };
template <> struct Words<4, 4> { typedef unsigned type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Words<4, 16> { typedef unsigned type __attribute__((ext_vector_type(4))); };

// The lanes of a workgroup over its rows: G of them share a row, vector j of a lane begins at column col(j).  A tensor's address is that of the workgroup's
// first row, the same for all lanes, and an offset of 32 bits that does not change from row to row.  A short vector is read from `width - V` on and moved down by what it
// overlaps, so that its lane takes no way of its own (which would wait for each load by itself).
template <typename S>
struct RowLanes {
    static constexpr int V = S::V, kThreads = block_threads(S::GC);
    static constexpr bool even = S::LIE == kEven;
    int G, lane, group, width;
    __device__ __forceinline__ RowLanes(int g, int w) : G(S::GC ? S::GC : g), lane(threadIdx.x & (G - 1)), group(threadIdx.x / G), width(w) {}
    __device__ __forceinline__ int rows() const { return kThreads / G; }
    __device__ __forceinline__ int col(int j) const { return (lane + j * G) * V; }
    __device__ __forceinline__ bool in(int j) const { return col(j) < width; }
    __device__ __forceinline__ int from(int j) const { return S::LIE == kUneven ? min(col(j), width - V) : col(j); }
    // the row's address (vectors then lie at col(j))
    template <typename T> __device__ __forceinline__ T* row(void* base, int64_t row0) const {
        return reinterpret_cast<T*>(static_cast<char*>(base) + row0 * width * sizeof(T) + (unsigned)(group * width * (int)sizeof(T)));
    }
    // V elements at `p`, the row's column from(j)
    template <typename T> __device__ __forceinline__ void words(const char* p, int j, unsigned (&w)[V * sizeof(T) / 4]) const {
        constexpr int bytes = V * sizeof(T), N = bytes / 4;
        if constexpr (S::LIE == kNarrow) {
#pragma unroll
            for (int k = 0; k < N; ++k) w[k] = 0;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (e >= width) break;
                if constexpr (sizeof(T) == 4) w[e] = reinterpret_cast<const unsigned*>(p)[e];
                else if constexpr (sizeof(T) == 2) w[e / 2] |= (unsigned)reinterpret_cast<const bf16_t*>(p)[e] << (16 * (e & 1));
                else w[e / 4] |= (unsigned)reinterpret_cast<const uint8_t*>(p)[e] << (8 * (e & 3));
            }
        } else {
            // (with the hint that no line is read again)
            const auto t = __builtin_nontemporal_load(reinterpret_cast<const typename Words<N, even ? bytes : (int)sizeof(T)>::type*>(p));
            __builtin_memcpy(w, &t, bytes);
        }
    }
    // Vector j of the lane's row as it lies in memory, and what is left to do with it.
    template <typename T> __device__ __forceinline__ void fetch(const void* base, int64_t row0, int j, unsigned (&w)[V * sizeof(T) / 4]) const {
        words<T>(static_cast<const char*>(base) + row0 * width * sizeof(T) + (unsigned)((group * width + from(j)) * (int)sizeof(T)), j, w);
    }
    template <typename T> __device__ __forceinline__ void align(int j, unsigned (&w)[V * sizeof(T) / 4]) const {
        if constexpr (S::LIE == kUneven) move_down<sizeof(T)>(w, (col(j) - from(j)) * (int)sizeof(T));
    }
    template <typename T> __device__ __forceinline__ void values(int j, RawCols<T, V>& w, float (&v)[V]) const {
        align<T>(j, w);
        raw_values<T, V>(w, v);
    }
    // Vector j of a row of fp32 that all rows share.  A lane that has no column there reads the row's last vector.
    __device__ __forceinline__ void shared(const float* p, int j, float (&v)[V]) const {
        if constexpr (even) {
            load_cols<V>(p + min(col(j), width - V), v);
        } else if constexpr (S::LIE == kUneven) {
            RawCols<float, V> w;
            __builtin_memcpy(w, p + from(j), sizeof(w));
            move_down<sizeof(float)>(w, min(col(j) - from(j), V - 1) * (int)sizeof(float));
            raw_values<float, V>(w, v);
        } else {
            load_v<false>(p, col(j), width, v);
        }
    }
    __device__ __forceinline__ unsigned fetch_scale(const uint8_t* scales, int64_t row0, int j) const {
        const int nb = held_blocks(width);
        return (scales + row0 * nb)[(unsigned)(group * nb + col(j) / kHeldBlock)];
    }
    // the type of the lane's row; negative: it stands for nothing
    __device__ __forceinline__ int type(const BlockParams& p, int64_t row0, int64_t rows) const {
        if (row0 + group >= rows) return -1;
        if (!p.types) return 0;
        const int t = (p.types + row0)[(unsigned)group];
        return (unsigned)t < (unsigned)p.T ? t : -1;
    }
};

size_t block_bwd_workspace(const rgnn_block_norm_desc_t* d);
rgnn_status_t block_bwd_rows8(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, const BlockBwdArgs& a, hipStream_t st);
rgnn_status_t block_bwd(const rgnn_block_norm_desc_t* d, BlockBwdArgs a, bool held, void* workspace, hipStream_t st);

}  // namespace rgnn
