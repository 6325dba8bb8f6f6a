// Rows in the registers of the lanes that share them: loads and stores of any width, sums over a row.  Internal.
#pragma once
#include "row_ops.h"

namespace rgnn {

constexpr int kBlock = 512;              // threads of a workgroup

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

// V elements as they lie in memory, for rows that are on their way while others are worked on.
template <typename T, int V> using RawCols = unsigned[V * sizeof(T) / 4];
template <typename T, int V>
__device__ __forceinline__ void raw_values(const RawCols<T, V>& w, float (&v)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e)
        v[e] = __uint_as_float(sizeof(T) == 4 ? w[e * sizeof(T) / 4] : e % 2 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
}
// Moves the elements of SIZE bytes in words down by `bytes`, fewer than there are, zeros after them.  (Lanes past a row's end come with zeros and any `bytes`: a shift
// is defined for them too.)
template <int SIZE, int N>
__device__ __forceinline__ void move_down(unsigned (&w)[N], int bytes) {
    if constexpr (N == 1) {
        w[0] >>= 8 * (bytes & 3);
    } else if constexpr (N == 2) {
        const unsigned long long v = ((unsigned long long)w[1] << 32 | w[0]) >> (8 * (bytes & 7));
        w[0] = (unsigned)v;
        w[1] = (unsigned)(v >> 32);
    } else {
        static_assert(SIZE >= 2, "halves of words at least");
#pragma unroll
        for (int k = 1; k < N; k *= 2)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const unsigned here = w[i], there = i + k < N ? w[i + k < N ? i + k : 0] : 0u;       // (values: a choice between places would put w into memory)
                w[i] = bytes & (4 * k) ? there : here;
            }
        if constexpr (SIZE == 2) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const unsigned here = w[i], there = i + 1 < N ? w[i + 1 < N ? i + 1 : 0] : 0u;
                w[i] = bytes & 2 ? here >> 16 | there << 16 : here;
            }
        }
    }
}

// Sum over the G lanes of a row (G a power of two up to 64), or over the workgroup.
__device__ __forceinline__ float lanes_sum(float v, int G) {
    if (G >= 2) v += dpp_move<kDppQuadSwap1>(v);
    if (G >= 4) v += dpp_move<kDppQuadSwap2>(v);
    if (G >= 8) v += dpp_move<kDppHalfMirror>(v);
    if (G >= 16) v += dpp_move<kDppMirror>(v);
    if (G >= 32) v = half_rows_sum(v);
    if (G >= 64) v = halves_sum(v);
    return v;
}

// Sum over a wavefront's lanes of the same number modulo G.
__device__ __forceinline__ float groups_sum(float v, int G) {
    if (G <= 1) v += dpp_move<kDppQuadSwap1>(v);
    if (G <= 2) v += dpp_move<kDppQuadSwap2>(v);
    if (G <= 4) v += dpp_move<kDppRowRotate + 4>(v);
    if (G <= 8) v += dpp_move<kDppRowRotate + 8>(v);
    if (G <= 16) v = half_rows_sum(v);
    if (G <= 32) v = halves_sum(v);
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

// One sum.
__device__ __forceinline__ void row_sum(float& a, int G, float* lds, int turn) {
    a = lanes_sum(a, min(G, 64));
    if (G <= 64) return;
    constexpr int W = kBlock / 64;
    float* const at = lds + (turn & 1) * 2 * W;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = a;
    __syncthreads();
    a = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) a += at[i];
}

// What a row's values are multiplied by where their squares' sum is infinite.  Any finite row's sum is in range then, 2^-32 or more, and the squares
// that vanish are below 2^-149.
constexpr float kScaleDown = 0x1p-80f;

template <bool EVEN, typename T, int V>
__device__ __forceinline__ void put(T* row, int c, int width, const float (&v)[V], int accumulate) {
    float t[V];
    zero_cols<V>(t);
    if (accumulate) load_v<EVEN>(row, c, width, t);
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] += v[e];
    store_v<EVEN>(row, c, width, t);
}

}  // namespace rgnn
