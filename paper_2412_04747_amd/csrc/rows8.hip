// Rows into 8 bits and back (rows8.h has the format).
//
// Five and three operations per value against 5 bytes (fp32) or 3 (bf16): the memory's rate is the bound.  A lane takes 16 bytes of x, and eight lanes
// (bf16: four) a block of 32 columns, whose largest value they find by lane moves.  Against 5.0 TB/s of a large copy: 2M rows of 128, bf16, packed in 113 us
// (6.9 TB/s) and unpacked in 116; 1M rows of 64, fp32, 51 and 45; 100003 rows of 349, fp32, 35 and 36, bf16, 26 and 28.  A workgroup for each 512 vectors, two per
// lane; 8192 workgroups that take several turns of four vectors: 116 and 127 us.  Rows narrower than a block leave lanes idle, as each takes a whole block's: 2M rows of 9, fp32, 50 and 44 us
// (1.8 and 2.1 TB/s), bf16 35 and 26 (1.6, 2.1); of 17, fp32, 51 and 54 (3.3, 3.2), bf16 37 and 34 (2.8, 3.0).
#include "rgnn_internal.h"
#include "device_utils.h"
#include "rows8.h"

namespace rgnn {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxGrid = 65536;
constexpr int kInFlight = 2;             // vectors that a lane has on their way

struct Rows8Args {
    int64_t rows;
    int width;
    int vectors;             // of a row, its last block filled up
    int64_t total;           // rows * vectors
    int streaming;           // what is written is more than the caches hold
    const void* x; int8_t* codes; uint8_t* scales;      // (unpack: x is written)
};

// Vector `base + at` of all rows, at below kThreads * kInFlight: its row and first column.  (FLAT below: rows are whole blocks, so that they are one long one.)  A vector
// that the row's end cuts is read from `from` on and moved down by what lies before it, so that no lane takes a way of its own.
template <int V>
struct Place {
    int64_t row;
    int c, from;
    __device__ __forceinline__ Place(const Rows8Args& a, int64_t row0, int rest, int at) {
        const int i = rest + at, q = (int)(((float)i + 0.5f) * (1.f / (float)a.vectors));      // (i below 2^13: exact)
        row = min(row0 + q, a.rows - 1);
        c = (i - q * a.vectors) * V;
        from = min(c, a.width - V);
    }
};

template <typename T, bool FLAT>
__global__ __launch_bounds__(kThreads) void rows8_pack_kernel(Rows8Args a) {
    constexpr int V = 16 / sizeof(T), LANES = kHeldBlock / V;
    const T* const x = static_cast<const T*>(a.x);
    const int nb = held_blocks(a.width);
    for (int64_t base = (int64_t)blockIdx.x * kThreads * kInFlight; base < a.total; base += (int64_t)gridDim.x * kThreads * kInFlight) {
        const int64_t row0 = FLAT ? 0 : base / a.vectors;
        const int rest = FLAT ? 0 : (int)(base - row0 * a.vectors);
        float v[kInFlight][V];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const int at = u * kThreads + threadIdx.x;
            if constexpr (FLAT) {
                load_cols_nt<V>(x + min(base + at, a.total - 1) * V, v[u]);
            } else {
                const Place<V> p(a, row0, rest, at);
                if (a.width < V) {
                    load_v<false>(x + p.row * a.width, p.c, a.width, v[u]);
                } else {
                    RawCols<T, V> w;
                    __builtin_memcpy(w, x + p.row * a.width + p.from, sizeof(w));
                    move_down<sizeof(T)>(w, min(p.c - p.from, V - 1) * (int)sizeof(T));
                    raw_values<T, V>(w, v[u]);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[u][e] = p.c < a.width ? v[u][e] : 0.f;       // (a vector of the last block that has no column)
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const int at = u * kThreads + threadIdx.x;
            const unsigned b = scale_byte(lanes_max(bits_max(v[u]), LANES));
            CodeWords<V> w;
            to_codes(v[u], b, w);
            if (base + at >= a.total) continue;
            if constexpr (FLAT) {
                store_codes<true, V>(a.codes + (base + at) * V, 0, V, w);
                if (at % LANES == 0) a.scales[(base + at) / LANES] = (uint8_t)b;
            } else {
                const Place<V> p(a, row0, rest, at);
                store_codes<false, V>(a.codes + p.row * a.width, p.c, a.width, w);
                if (p.c % kHeldBlock == 0) a.scales[p.row * nb + p.c / kHeldBlock] = (uint8_t)b;
            }
        }
    }
}

template <typename T, bool FLAT>
__global__ __launch_bounds__(kThreads) void rows8_unpack_kernel(Rows8Args a) {
    constexpr int V = 16 / sizeof(T), LANES = kHeldBlock / V;
    T* const x = static_cast<T*>(const_cast<void*>(a.x));
    const int nb = held_blocks(a.width);
    for (int64_t base = (int64_t)blockIdx.x * kThreads * kInFlight; base < a.total; base += (int64_t)gridDim.x * kThreads * kInFlight) {
        const int64_t row0 = FLAT ? 0 : base / a.vectors;
        const int rest = FLAT ? 0 : (int)(base - row0 * a.vectors);
        CodeWords<V> w[kInFlight];
        unsigned b[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const int at = u * kThreads + threadIdx.x;
            if constexpr (FLAT) {
                const int64_t i = min(base + at, a.total - 1);
                load_codes<true, V>(a.codes + i * V, 0, V, w[u]);
                b[u] = a.scales[i / LANES];
            } else {
                const Place<V> p(a, row0, rest, at);
                if (V == 4 || a.width < V) {         // (four codes: 36 us, 43 the other way, 100003 rows of 349)
                    load_codes<false, V>(a.codes + p.row * a.width, min(p.c, a.width - 1), a.width, w[u]);
                } else {
                    __builtin_memcpy(w[u], a.codes + p.row * a.width + p.from, V);
                    move_down<1>(w[u], min(p.c - p.from, V - 1));
                }
                b[u] = a.scales[p.row * nb + p.c / kHeldBlock];
            }
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const int at = u * kThreads + threadIdx.x;
            float v[V];
            from_codes<V>(w[u], held_step(b[u]), v);
            if (base + at >= a.total) continue;
            if constexpr (FLAT) {
                if (a.streaming) store_cols_nt<V>(x + (base + at) * V, v);
                else store_cols<V>(x + (base + at) * V, v);
            } else {
                const Place<V> p(a, row0, rest, at);
                store_v<false>(x + p.row * a.width, p.c, a.width, v);
            }
        }
    }
}

rgnn_status_t check(const rgnn_rows8_desc_t* d, const void* x, const rgnn_rows8_t* r) {
    if (!d) RGNN_FAIL(RGNN_EINVAL, "desc is NULL");
    RGNN_TRY(check_rows(d->rows));
    if (d->width < 1) RGNN_FAIL(RGNN_EINVAL, "width %d is not positive", d->width);
    if (d->width > 8192) RGNN_FAIL(RGNN_EUNSUPPORTED, "width %d not supported (up to 8192)", d->width);
    RGNN_TRY(check_dtype(d->dtype));
    if (d->rows == 0) return RGNN_OK;
    if (!x || !r || !r->codes || !r->scales) RGNN_FAIL(RGNN_EINVAL, "x, codes or scales is NULL");
    const Span xs = span(x, (size_t)d->rows * d->width, d->dtype), cs = code_span(r, d->rows, d->width), ss = scale_span(r, d->rows, d->width);
    RGNN_TRY(check_aligned(xs));
    RGNN_TRY(check_aligned(cs));
    if (xs.overlaps(cs) || xs.overlaps(ss) || cs.overlaps(ss)) RGNN_FAIL(RGNN_EINVAL, "x, codes and scales overlap");
    return RGNN_OK;
}

template <typename F>
rgnn_status_t launch(const rgnn_rows8_desc_t* d, const void* x, const rgnn_rows8_t* r, F f) {
    const int v = d->dtype == RGNN_BF16 ? 8 : 4, vectors = held_blocks(d->width) * (kHeldBlock / v);
    const Rows8Args a{d->rows, d->width, vectors, d->rows * vectors, d->rows * d->width * (d->dtype == RGNN_BF16 ? 2 : 4) > kCachedBytes, x, r->codes, r->scales};
    const unsigned grid = (unsigned)std::min<int64_t>(kMaxGrid, (a.total + kThreads * kInFlight - 1) / (kThreads * kInFlight));
    f(a, grid, d->width % kHeldBlock == 0);
    RGNN_CHECK_LAUNCH();
    return RGNN_OK;
}

}  // namespace

}  // namespace rgnn

using namespace rgnn;

extern "C" rgnn_status_t rgnn_rows8_pack(const rgnn_rows8_desc_t* desc, const void* x, const rgnn_rows8_t* to, void* stream) {
    RGNN_TRY(check(desc, x, to));
    if (desc->rows == 0) return RGNN_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return launch(desc, x, to, [&](const Rows8Args& a, unsigned grid, bool flat) {
        KernelTimer timer(st, "rows8_pack");
        if (desc->dtype == RGNN_BF16) flat ? rows8_pack_kernel<bf16_t, true><<<grid, kThreads, 0, st>>>(a) : rows8_pack_kernel<bf16_t, false><<<grid, kThreads, 0, st>>>(a);
        else flat ? rows8_pack_kernel<float, true><<<grid, kThreads, 0, st>>>(a) : rows8_pack_kernel<float, false><<<grid, kThreads, 0, st>>>(a);
    });
}

extern "C" rgnn_status_t rgnn_rows8_unpack(const rgnn_rows8_desc_t* desc, const rgnn_rows8_t* from, void* x, void* stream) {
    RGNN_TRY(check(desc, x, from));
    if (desc->rows == 0) return RGNN_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return launch(desc, x, from, [&](const Rows8Args& a, unsigned grid, bool flat) {
        KernelTimer timer(st, "rows8_unpack");
        if (desc->dtype == RGNN_BF16) flat ? rows8_unpack_kernel<bf16_t, true><<<grid, kThreads, 0, st>>>(a) : rows8_unpack_kernel<bf16_t, false><<<grid, kThreads, 0, st>>>(a);
        else flat ? rows8_unpack_kernel<float, true><<<grid, kThreads, 0, st>>>(a) : rows8_unpack_kernel<float, false><<<grid, kThreads, 0, st>>>(a);
    });
}
