// What the operators on rows (norm, feed-forward block, gradient clipping) share: checks of their arguments, and elements of either type.  Internal.
#pragma once
#include "rgnn_internal.h"
#include "device_utils.h"

namespace rgnn {

// A tensor argument's bytes.  An empty or absent one overlaps nothing.
struct Span {
    const char* p;
    size_t bytes;
    bool overlaps(const Span& o) const { return p && o.p && bytes && o.bytes && p < o.p + o.bytes && o.p < p + bytes; }
    bool same(const Span& o) const { return p == o.p && bytes == o.bytes; }
};
inline Span span(const void* p, size_t n, int32_t dtype) { return Span{static_cast<const char*>(p), n * (dtype == RGNN_BF16 ? 2 : 4)}; }

inline rgnn_status_t check_aligned(const Span& s) {
    if (reinterpret_cast<uintptr_t>(s.p) % 16) RGNN_FAIL(RGNN_EINVAL, "a tensor is not 16-byte aligned");
    return RGNN_OK;
}
inline rgnn_status_t check_dtype(int32_t t) {
    if (t != RGNN_F32 && t != RGNN_BF16) RGNN_FAIL(RGNN_EINVAL, "unknown dtype %d", t);
    return RGNN_OK;
}
inline rgnn_status_t check_rows(int64_t rows) {
    if (rows < 0) RGNN_FAIL(RGNN_EINVAL, "rows %lld is negative", (long long)rows);
    if (rows > INT32_MAX) RGNN_FAIL(RGNN_EUNSUPPORTED, "rows %lld not supported (below 2^31)", (long long)rows);
    return RGNN_OK;
}

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return __uint_as_float((unsigned)v << 16); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t narrow<bf16_t>(float v) { return (bf16_t)(bf16_pack2(v, v) & 0xFFFFu); }

}  // namespace rgnn
