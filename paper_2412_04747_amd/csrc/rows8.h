// Rows in 8 bits: every 32 columns of a row share a scale byte b, a value is code 2^(b - 133) with a code of -127 .. 127.  Internal.
//
// With m the largest absolute value of the 32 and 2^e <= m < 2^(e + 1), a step is 2^(e - 6), or twice that where m would round to 128 steps; b = e + 127 (+ 1).
// So a code is off by at most half a step, and neither x / step nor code * step is rounded: a code depends on x alone, and its value, 7 bits and a power of
// two, is exact in fp32 and in bfloat16 (one plane of the matrix instructions' operands).
// Steps stop at 2^-126 (b = 7), the least normal number; at the other end b stops at 254, where codes stop at 127.  An infinity or NaN makes its 32 columns
// b = 255, which stands for NaN.  Scale bytes below 7, which nothing here writes, stand for zeros.
#pragma once
#include "row_cols.h"

namespace rgnn {

constexpr int kHeldBlock = 32;           // columns that share a scale
inline __host__ __device__ int held_blocks(int width) { return (width + kHeldBlock - 1) / kHeldBlock; }

// Largest of the bit patterns of absolute values over the lanes that hold a block (N of them, or all G of a narrower row).
__device__ __forceinline__ unsigned lanes_max(unsigned v, int n) {
    auto with = [&](int other) { v = max(v, (unsigned)other); };
    if (n >= 2) with(dpp_move<kDppQuadSwap1>((int)v));
    if (n >= 4) with(dpp_move<kDppQuadSwap2>((int)v));
    if (n >= 8) with(dpp_move<kDppHalfMirror>((int)v));
    return v;
}
template <int V>
__device__ __forceinline__ unsigned bits_max(const float (&v)[V]) {
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    return m;
}
// (127.5 / 64 = 1 + 0x7F0000 2^-23: from there on the sum below carries into the exponent)
__device__ __forceinline__ unsigned scale_byte(unsigned m) { return m >= 0x7F800000u ? 255u : min(max((m + 0x10000u) >> 23, 7u), 254u); }

template <int V> using CodeWords = unsigned[V / 4];
// Codes of V values, four to a word.  Added to 1.5 2^23 a value is rounded to nearest even, and its last byte is the code.
template <int V>
__device__ __forceinline__ void to_codes(const float (&v)[V], unsigned b, CodeWords<V>& w) {
    const float by = __uint_as_float((260u - b) << 23);            // 2^(133 - b)
    unsigned q[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        q[e] = __float_as_uint(fminf(fmaxf(v[e] * by, -127.f), 127.f) + 12582912.f) & 255u;
        q[e] = b == 255u ? 0u : q[e];
    }
#pragma unroll
    for (int k = 0; k < V / 4; ++k) w[k] = q[4 * k] | q[4 * k + 1] << 8 | q[4 * k + 2] << 16 | q[4 * k + 3] << 24;
}
__device__ __forceinline__ float held_step(unsigned b) { return b == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float((max(b, 6u) - 6u) << 23); }
template <int V>
__device__ __forceinline__ void from_codes(const CodeWords<V>& w, float step, float (&v)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = (float)((int)(w[e / 4] << (24 - 8 * (e & 3))) >> 24) * step;
}

// V codes from a row's column c on, those before `width` (EVEN as in load_v).
template <bool EVEN, int V>
__device__ __forceinline__ void load_codes(const int8_t* row, int c, int width, CodeWords<V>& w) {
    if (EVEN || c + V <= width) {
        __builtin_memcpy(w, EVEN ? static_cast<const int8_t*>(__builtin_assume_aligned(row + c, V)) : row + c, V);
    } else {
#pragma unroll
        for (int k = 0; k < V / 4; ++k) {
            w[k] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + 4 * k + e < width) w[k] |= (unsigned)(uint8_t)row[c + 4 * k + e] << (8 * e);
        }
    }
}
template <bool EVEN, int V>
__device__ __forceinline__ void store_codes(int8_t* row, int c, int width, const CodeWords<V>& w) {
    if (EVEN || c + V <= width) {
        __builtin_memcpy(EVEN ? static_cast<int8_t*>(__builtin_assume_aligned(row + c, V)) : row + c, w, V);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < width) row[c + e] = (int8_t)(w[e / 4] >> (8 * (e & 3)));
    }
}

// The tensors of rows in 8 bits as arguments.
inline Span code_span(const rgnn_rows8_t* r, int64_t rows, int width) { return Span{reinterpret_cast<const char*>(r->codes), (size_t)rows * width}; }
inline Span scale_span(const rgnn_rows8_t* r, int64_t rows, int width) { return Span{reinterpret_cast<const char*>(r->scales), (size_t)rows * held_blocks(width)}; }

}  // namespace rgnn
