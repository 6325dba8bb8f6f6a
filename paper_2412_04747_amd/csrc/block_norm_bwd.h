// The junction of a block's output with the residual stream, backward (block_norm.h has the formulas): the rows' kernel, which block_norm_bwd.hip and
// block_norm_held.hip (a and s in 8 bits) launch.  Internal.
//
// Some 36 operations per element against 12 to 24 bytes: the memory's rate is the bound.  a and s come as they are or in 8 bits; the sum and both reciprocal roots
// are formed again from them, in the registers of the lanes that hold the row: three sums over the row follow each other, and each tensor is passed once.
// Sums over rows: a lane keeps its columns' G and dw2 in registers while its rows have one type.  Where the type changes it adds G to the place of
// that type in the LDS, which is its wavefront's (lanes of one wavefront that share columns take turns), so that no order depends on timing.  Nodes are
// mostly stored type by type: then that is rare.  A workgroup leaves one partial row per type; a second launch adds those in order.
// Against 4.9 TB/s of a large copy: 1M rows of 64, fp32, four types, 272 us (5.7 TB/s; from 8 bits 212, 5.5; in mixed order 282); 2M rows of 128, bf16, 562 (5.5; from
// 8 bits 463, 5.6); 30011 rows of 349, fp32, 65 (3.8), seven mixed types 82; bf16, by vectors of four columns too,
// 45 and 60 (2.8, 2.1); 100000 from 8 bits, fp32, 185 and 261 (3.4, 2.4).  Without norms, 1M rows of 64, four mixed types, 265 (4.9).  Before the next row's
// tensors were fetched while a row is worked on, and the addresses had 32 bits of their own, the same kernel took 1000 us for 2M rows of 128 from 8 bits.
#pragma once
#include <float.h>

#include "rgnn_internal.h"
#include "device_utils.h"
#include "block_norm.h"

namespace rgnn {

namespace {

// Wavefronts that share a SIMD.  With the next row's tensors on their way three are enough, and more only spread what is read at a time: the registers of 4 columns per
// lane would allow four (1M rows of 64, fp32: 314 us with four, 301 with three; of 8 columns, from 8 bits: 520 with three, 545 with two).
constexpr int per_simd(int cols, int GC) { return GC == kBlock || cols > 8 ? 2 : 3; }
constexpr size_t kLdsBytes = 160 * 1024;      // of a compute unit
constexpr int kSumsLds = 4 * (kBlock / 64);
constexpr int kTail = kBlock / 64;       // places behind a type's columns in the LDS: shares of dscale

// A type's place: its columns, filled up to whole vectors of four, then shares of dscale.  In a workgroup's partial rows the shares are one (of four).
__host__ __device__ inline int columns4(int width) { return (width + 3) / 4 * 4; }
__host__ __device__ inline int place_len(int width) { return columns4(width) + kTail; }
__host__ __device__ inline int part_len(int width) { return columns4(width) + 4; }
// Partial rows lie by groups of columns: [group][workgroup][T + 1][kReduceCols].
constexpr int kReduceCols = 8;
__host__ __device__ inline int part_groups(int width) { return (part_len(width) + kReduceCols - 1) / kReduceCols; }

// i / n for i below 2^16 and a positive n
__device__ __forceinline__ int quotient(int i, int n) { return (int)(((float)i + 0.5f) * (1.f / (float)n)); }

// The parameters' gradients of columns c0 .. c0 + n - 1 of the partial rows' sums, by all threads of a workgroup.  at(t, c - c0): the place in the LDS of G[t], for
// t = T of dw2; the column behind the last vector holds dscale.
template <typename F>
__device__ __forceinline__ void finish(const BlockBwdArgs& a, int c0, int n, int threads, F at) {
    const int T = a.p.T;
    auto give = [&](float* p, float v) { *p = a.accumulate ? v + *p : v; };
    for (int i = threadIdx.x; i < (T + 1) * n; i += threads) {
        const int t = quotient(i, n), c = c0 + i - t * n;
        float& g = at(t, c - c0);
        if (c >= a.width) {
            if (c == columns4(a.width) && t < T && a.grads.scale) give(a.grads.scale + t, g);
        } else if (t == T) {
            if (a.grads.w_before) give(a.grads.w_before + c, g);
        } else {
            if (a.grads.gate) give(a.grads.gate + t * a.width + c, (a.p.w1 ? a.p.w1[c] : 1.f) * g);
            if (a.p.gate) g *= a.p.gate[t * a.width + c];
        }
    }
    if (!a.grads.w_after) return;
    __syncthreads();
    for (int k = threadIdx.x; k < n && c0 + k < a.width; k += threads) {
        float v = 0.f;
        for (int t = 0; t < T; ++t) v += at(t, k);
        give(a.grads.w_after + c0 + k, v);
    }
}

template <typename TA, typename TS, typename TO, typename S, bool HELD>
__global__ __launch_bounds__(block_threads(S::GC), per_simd(S::V * S::NV, S::GC)) void block_bwd_kernel(BlockBwdArgs a) {
    extern __shared__ float lds[];           // row_sums' halves, then the places of the types
    constexpr int V = S::V, NV = S::NV, kThreads = block_threads(S::GC);
    constexpr bool WIDE = S::GC == kBlock, AHEAD = V * NV <= 8, EVEN = S::LIE == kEven, STEPS = HELD && EVEN;
    constexpr int kWaves = kThreads / 64, slots = WIDE ? 1 : kWaves;
    const RowLanes<S> sh(a.G, a.width);
    const float inv = 1.f / (float)a.width;
    const int T = a.p.T, len = place_len(a.width), wave = threadIdx.x >> 6;
    float* const places = lds + kSumsLds;
    float* const mine = places + (WIDE ? 0 : wave * (T + 1) * len);
    if (a.sums) {
        for (int i = threadIdx.x; i < slots * (T + 1) * (len / 4); i += kThreads) reinterpret_cast<float4*>(places)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        __syncthreads();
    }
    // gw: gate w1 of the type at hand
    float w2[NV][V], gw[NV][V], dw2[NV][V], G[NV][V], dscale = 0.f, scale = 1.f;
    auto load_type = [&](int t) {
        scale = a.p.scale ? a.p.scale[t] : 1.f;
        float w[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) gw[j][e] = w[j][e] = 1.f;
        // (lanes past the row's end load its last vector: all loads are on their way together)
        if (a.p.gate)
#pragma unroll
            for (int j = 0; j < NV; ++j) sh.shared(a.p.gate + (unsigned)(t * a.width), j, gw[j]);
        if (a.p.w1)
#pragma unroll
            for (int j = 0; j < NV; ++j) sh.shared(a.p.w1, j, w[j]);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) gw[j][e] = sh.in(j) ? gw[j][e] * w[j][e] : 0.f;
    };
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        zero_cols<V>(dw2[j]);
        zero_cols<V>(G[j]);
        zero_cols<V>(w2[j]);
        if (a.p.w2 && sh.in(j)) sh.shared(a.p.w2, j, w2[j]);
    }
    load_type(0);
    // adds a lane's sums to place t of its wavefront (workgroup); the lanes with `who`, those of a row together
    auto give = [&](bool who, int t, float (&v)[NV][V], float& tail) {
        float sum = lanes_sum(tail, min(sh.G, 64));
        float* const at = mine + t * len;
        auto add = [&]() {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (sh.in(j)) {
                    float o[V];
                    load_cols<V>(at + sh.col(j), o);
#pragma unroll
                    for (int e = 0; e < V; ++e) o[e] += v[j][e];
                    store_cols<V>(at + sh.col(j), o);
                }
                zero_cols<V>(v[j]);
            }
            if ((sh.lane & 63) == 0) at[len - kTail + (WIDE ? wave : 0)] += sum;
            tail = 0.f;
        };
        if (sh.G >= 64) {
            if (who) add();
            return;
        }
        const unsigned long long which = __ballot(who);
        if (which == ~0ull && __all(t == __builtin_amdgcn_readfirstlane(t))) {       // all of one type: their sum in one turn
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) v[j][e] = groups_sum(v[j][e], sh.G);
            sum = groups_sum(sum, sh.G);
            if ((threadIdx.x & 63) < (unsigned)sh.G) add();
#pragma unroll
            for (int j = 0; j < NV; ++j) zero_cols<V>(v[j]);
            tail = 0.f;
            return;
        }
        for (int k = 0; k < 64; k += sh.G) {
            if (!((which >> k) & 1)) continue;
            if ((threadIdx.x & 63 & ~(sh.G - 1)) == (unsigned)k) add();
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    // A row's tensors as they lie in memory: the next row's are on their way while a row is worked on, and its type is known before.
    RawCols<TA, V> xr[NV];
    RawCols<TS, V> sr[NV], dsr[NV];
    RawCols<TO, V> dyr[NV];
    CodeWords<V> xc[NV], sc[NV];
    unsigned xb[NV], sb[NV];
    auto clear_words = [](auto& w) {
#pragma unroll
        for (int k = 0; k < (int)(sizeof(w) / 4); ++k) w[k] = 0;
    };
    auto fetch = [&](int64_t row0, int t) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if constexpr (HELD) {
                clear_words(xc[j]);
                clear_words(sc[j]);
                xb[j] = sb[j] = 0;
            } else {
                clear_words(xr[j]);
                clear_words(sr[j]);
            }
            clear_words(dyr[j]);
            clear_words(dsr[j]);
            if (t < 0 || !sh.in(j)) continue;
            if constexpr (HELD) {
                sh.template fetch<int8_t>(a.a, row0, j, xc[j]);
                sh.template fetch<int8_t>(a.s, row0, j, sc[j]);
                xb[j] = sh.fetch_scale(a.a_scales, row0, j);
                sb[j] = sh.fetch_scale(a.s_scales, row0, j);
            } else {
                sh.template fetch<TA>(a.a, row0, j, xr[j]);
                sh.template fetch<TS>(a.s, row0, j, sr[j]);
            }
            if (a.dy) sh.template fetch<TO>(a.dy, row0, j, dyr[j]);
            if (a.ds) sh.template fetch<TS>(a.ds, row0, j, dsr[j]);
        }
    };
    const int64_t step = (int64_t)gridDim.x * sh.rows();
    int turn = 0, type = a.p.types ? -1 : 0;
    int64_t row0 = (int64_t)blockIdx.x * sh.rows();
    int t = sh.type(a.p, row0, a.rows), next = AHEAD ? sh.type(a.p, row0 + step, a.rows) : 0;
    if constexpr (AHEAD) fetch(row0, t);
    // (the trip count is the same for all threads of a workgroup whose rows are its own: the barrier in row_sums)
    for (; row0 < a.rows; row0 += step) {
        if constexpr (!AHEAD) fetch(row0, t);
        // Rows in 8 bits: x and s are their codes, a lane's all with one step (xs, ss), which its scalars take up (not of short vectors: their registers are full).
        float x[NV][V], s[NV][V], dy[NV][V], dt[NV][V], xs[NV], ss[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            xs[j] = ss[j] = 1.f;
            if constexpr (HELD) {
                sh.template align<int8_t>(j, xc[j]);
                sh.template align<int8_t>(j, sc[j]);
                if constexpr (STEPS) {
                    xs[j] = held_step(xb[j]);
                    ss[j] = held_step(sb[j]);
                }
                from_codes<V>(xc[j], STEPS ? 1.f : held_step(xb[j]), x[j]);
                from_codes<V>(sc[j], STEPS ? 1.f : held_step(sb[j]), s[j]);
            } else {
                sh.template values<TA>(j, xr[j], x[j]);
                sh.template values<TS>(j, sr[j], s[j]);
            }
            sh.template values<TO>(j, dyr[j], dy[j]);
            sh.template values<TS>(j, dsr[j], dt[j]);
        }
        const int now = t;
        const bool live = row0 + sh.group < a.rows;
        if constexpr (AHEAD) {
            t = next;
            fetch(row0 + step, t);
            next = sh.type(a.p, row0 + 2 * step, a.rows);
        } else {
            t = sh.type(a.p, row0 + step, a.rows);
        }
        const bool change = now >= 0 && now != type;
        if (__any(change)) {
            if (a.sums) give(change && type >= 0, max(type, 0), G, dscale);
            if (change) {
                type = now;
                load_type(now);
            }
        }
        float q1 = 1.f, k1 = 1.f;
        if (a.p.w1) {
            float sq = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) sq += dot_cols<V>(x[j], x[j]) * xs[j] * xs[j];
            row_sum(sq, sh.G, lds, turn++);
            if (!(sq <= FLT_MAX)) {          // as in the forward; the scaled values take their place
                k1 = kScaleDown;
                sq = 0.f;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if constexpr (STEPS) {
                        xs[j] *= k1;
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e) x[j][e] *= k1;
                    }
                    sq += dot_cols<V>(x[j], x[j]) * xs[j] * xs[j];
                }
                row_sum(sq, sh.G, lds, turn++);
            }
            q1 = rsqrtf(sq * inv + a.eps * k1 * k1);
        }
        // x: from here on a q1
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const float by = STEPS ? q1 * xs[j] : q1;
#pragma unroll
            for (int e = 0; e < V; ++e) x[j][e] *= by;
        }
        if (a.dy) {
            float u[NV][V], sq = 0.f, gs = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const float by = STEPS ? scale * ss[j] : scale;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    u[j][e] = by * s[j][e] + x[j][e] * gw[j][e];
                    sq += u[j][e] * u[j][e];
                    gs += dy[j][e] * w2[j][e] * u[j][e];
                }
            }
            row_sums(sq, gs, sh.G, lds, turn++);
            float k2 = 1.f;
            if (!(sq <= FLT_MAX)) {
                k2 = kScaleDown;
                sq = gs = 0.f;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        u[j][e] *= k2;
                        sq += u[j][e] * u[j][e];
                        gs += dy[j][e] * w2[j][e] * u[j][e];
                    }
                row_sums(sq, gs, sh.G, lds, turn++);
            }
            // (with v = k u: q(u) = k q(v), u q(u)^2 mean(g u) = v q(v)^2 mean(g v); a row that stands for nothing has zeros here, with eps = 0 NaN)
            const float q2 = rsqrtf(sq * inv + a.eps * k2 * k2), along = q2 * q2 * (gs * inv), qk = q2 * k2;
            if (now >= 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        dt[j][e] += qk * (dy[j][e] * w2[j][e] - u[j][e] * along);
                        dw2[j][e] += dy[j][e] * (u[j][e] * q2);
                    }
            }
        }
        auto out = [&](auto* to, int j, const float (&v)[V]) {
            if constexpr (EVEN)
                if (a.streaming) return store_cols_nt<V>(to + sh.col(j), v);
            put<EVEN>(to, sh.col(j), a.width, v, a.accumulate);
        };
        TA* const da_row = sh.template row<TA>(a.da, row0);
        TS* const ds_row = sh.template row<TS>(a.dstream, row0);
        // dS, and what the row adds to its type's sums
        auto stream = [&]() {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (!sh.in(j)) continue;
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    v[e] = scale * dt[j][e];
                    G[j][e] += dt[j][e] * x[j][e];
                }
                dscale += dot_cols<V>(dt[j], s[j]) * ss[j];
                if (a.dstream) out(ds_row, j, v);
            }
        };
        // (dS before the last sum, which leaves h in dT's place; short vectors' stores take ways of their own, and once is enough)
        constexpr bool SOON = EVEN;
        if (SOON && now >= 0) stream();
        float along = 0.f;
        if (SOON || a.p.w1) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float h = dt[j][e] * gw[j][e];
                    along += h * x[j][e];
                    if constexpr (SOON) dt[j][e] = h;
                }
        }
        if (a.p.w1) {
            row_sum(along, sh.G, lds, turn++);
            along *= inv;
        } else {
            along = 0.f;
        }
        if (now >= 0) {
            const float qk = q1 * k1;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (!a.da || !sh.in(j)) continue;
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = qk * ((SOON ? dt[j][e] : dt[j][e] * gw[j][e]) - x[j][e] * along);
                out(da_row, j, v);
            }
            if (!SOON) stream();
        } else if (live && !a.accumulate) {
            float none[V];
            zero_cols<V>(none);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (!sh.in(j)) continue;
                if (a.da) out(da_row, j, none);
                if (a.dstream) out(ds_row, j, none);
            }
        }
    }
    if (!a.sums) return;
    // (lanes that never had a row hold zeros and go with the others)
    const unsigned long long with_rows = __ballot(type >= 0);
    if (with_rows) {
        const int any = __shfl(type, __ffsll((unsigned long long)with_rows) - 1);
        give(true, type >= 0 ? type : any, G, dscale);
    }
    float unused = 0.f;
    give(true, T, dw2, unused);
    __syncthreads();
    // the wavefronts' places in order
    const int L4 = part_len(a.width) / 4;
    for (int i = threadIdx.x; i < (T + 1) * L4; i += kThreads) {
        const int t = quotient(i, L4), c = 4 * (i - t * L4);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](const float4& o) { v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w; };
        for (int k = 0; k < slots; ++k) {
            const float4* const at = reinterpret_cast<const float4*>(places + (k * (T + 1) + t) * len + c);
            add(at[0]);
            if (c == L4 * 4 - 4) add(at[1]);
        }
        if (c == L4 * 4 - 4) v = make_float4(v.x + v.y + v.z + v.w, 0.f, 0.f, 0.f);
        // (each place's vectors are read by one lane alone, which may write there)
        if (gridDim.x > 1) *reinterpret_cast<float4*>(a.part + (((int64_t)(c / kReduceCols) * gridDim.x + blockIdx.x) * (T + 1) + t) * kReduceCols + c % kReduceCols) = v;
        else *reinterpret_cast<float4*>(places + t * len + c) = v;
    }
    if (gridDim.x > 1) return;
    __syncthreads();
    finish(a, 0, part_len(a.width), kThreads, [&](int t, int c) -> float& { return places[t * len + c]; });
}

inline size_t lds_bytes(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, bool sums) {
    // (four places of each type, (types + 1) * (width + 12) <= 9600 together: 154 KB at most; or one: 82)
    return sizeof(float) * (kSumsLds + (sums ? (size_t)(p.G == kBlock ? 1 : block_threads(p.G) / 64) * (d->types + 1) * place_len(d->width) : 0));
}
// As many as are resident at once, so that none comes in a second turn.  (What two turns of a workgroup finish is left to one: the sums then need no second launch.)
inline int workgroups(const rgnn_block_norm_desc_t* d) {
    const JunctionPlan p = block_plan(d);
    if (p.turns <= 2) return (int)std::min<int64_t>(p.turns, 1);
    const int waves = 4 * per_simd(p.V * p.NV, p.G) / (block_threads(p.G) / 64), room = (int)(kLdsBytes / lds_bytes(d, p, true));
    const int64_t most = 256 * std::max(1, std::min(waves, room));
    return (int)std::min(most, p.turns);
}

template <typename TA, typename TS, typename TO, bool HELD>
rgnn_status_t launch_rows(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, const BlockBwdArgs& a, hipStream_t st) {
    return block_with_shape<sizeof(TA) + sizeof(TS) + sizeof(TO) == 6>(d, p, [&](auto shape) -> rgnn_status_t {
        using S = decltype(shape);
        auto* const kernel = block_bwd_kernel<TA, TS, TO, S, HELD>;
        const size_t lds = lds_bytes(d, p, a.sums);
        RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds));
        KernelTimer timer(st, "block_norm_bwd");
        kernel<<<workgroups(d), block_threads(S::GC), lds, st>>>(a);
        RGNN_CHECK_LAUNCH();
        return RGNN_OK;
    });
}

// The rows' launch for all types of tensors.
template <bool HELD>
rgnn_status_t launch_types(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, const BlockBwdArgs& a, hipStream_t st) {
    return block_with_types(d, [&](auto ta, auto ts, auto to) { return launch_rows<decltype(ta), decltype(ts), decltype(to), HELD>(d, p, a, st); });
}

}  // namespace

}  // namespace rgnn
