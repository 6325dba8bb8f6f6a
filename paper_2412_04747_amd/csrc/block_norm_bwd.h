// The junction of a block's output with the residual stream, backward (block_norm.h has the formulas): the rows' kernel, which block_norm_bwd.hip and
// block_norm_held.hip (a and s in 8 bits) launch.  Internal.
//
// Some 36 operations per element against 12 to 24 bytes: the memory's rate is the bound.  a and s come as they are or in 8 bits; the sum and both reciprocal roots
// are formed again from them, in the registers of the lanes that hold the row: three sums over the row follow each other, and each tensor is passed once.
// Sums over rows: a lane keeps its columns' G and dw2 in registers while its rows have one type.  Where the type changes it adds G to the place of
// that type in the LDS, which is its wavefront's (lanes of one wavefront that share columns take turns), so that no order depends on timing.  Nodes are
// mostly stored type by type: then that is rare.  A workgroup leaves one partial row per type; a second launch adds those in order.
#pragma once
#include <float.h>

#include "rgnn_internal.h"
#include "device_utils.h"
#include "block_norm.h"

namespace rgnn {

namespace {

constexpr int kMaxBlocks = 512;
constexpr int kWaves = kBlock / 64;
constexpr int kTail = kWaves;            // places behind a type's columns in the LDS: shares of dscale

__host__ __device__ inline int place_len(int width) { return (width + 3) / 4 * 4 + kTail; }
__host__ __device__ inline int part_len(int T, int width) { return (T + 1) * (width + 1); }

// The parameters' gradients of column c (or, c = width, of the types' scales) from total(t): G[t] for t < T, dw2 for t = T.
template <typename F>
__device__ __forceinline__ void finish(const BlockBwdArgs& a, int c, F total) {
    const int T = a.p.T;
    if (c == a.width) {
        if (a.grads.scale)
            for (int t = 0; t < T; ++t) a.grads.scale[t] = total(t) + (a.accumulate ? a.grads.scale[t] : 0.f);
        return;
    }
    const float w = a.p.w1 ? a.p.w1[c] : 1.f;
    float dw = 0.f;
    for (int t = 0; t < T; ++t) {
        const float g = total(t);
        const int64_t at = (int64_t)t * a.width + c;
        dw += (a.p.gate ? a.p.gate[at] : 1.f) * g;
        if (a.grads.gate) a.grads.gate[at] = w * g + (a.accumulate ? a.grads.gate[at] : 0.f);
    }
    if (a.grads.w_after) a.grads.w_after[c] = dw + (a.accumulate ? a.grads.w_after[c] : 0.f);
    if (a.grads.w_before) a.grads.w_before[c] = total(T) + (a.accumulate ? a.grads.w_before[c] : 0.f);
}

template <typename TA, typename TS, typename TO, int V, int NV, bool EVEN, bool HELD>
__global__ __launch_bounds__(kBlock) void block_bwd_kernel(BlockBwdArgs a) {
    extern __shared__ float lds[];           // row_sums' halves, then the places of the types
    const Shape sh(a.G);
    const float inv = 1.f / (float)a.width;
    const int T = a.p.T, len = place_len(a.width), slots = a.G > 64 ? 1 : kWaves, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float* const places = lds + 4 * kWaves;
    float* const mine = places + (a.G > 64 ? 0 : wave * (T + 1) * len);
    if (a.sums) {
        for (int i = threadIdx.x; i < slots * (T + 1) * len; i += kBlock) places[i] = 0.f;
        __syncthreads();
    }
    float w1[NV][V], w2[NV][V], gate[NV][V], dw2[NV][V], G[NV][V], dscale = 0.f, scale = a.p.scale ? a.p.scale[0] : 1.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (sh.lane + j * sh.G) * V;
        zero_cols<V>(dw2[j]);
        zero_cols<V>(G[j]);
#pragma unroll
        for (int e = 0; e < V; ++e) w1[j][e] = w2[j][e] = gate[j][e] = 1.f;
        if (c < a.width) {
            if (a.p.w1) load_v<EVEN>(a.p.w1, c, a.width, w1[j]);
            if (a.p.w2) load_v<EVEN>(a.p.w2, c, a.width, w2[j]);
            if (a.p.gate) load_v<EVEN>(a.p.gate, c, a.width, gate[j]);
        }
    }
    // adds a lane's sums to place t of its wavefront (workgroup); the lanes with `who`, those of a row together
    auto give = [&](bool who, int t, float (&v)[NV][V], float& tail) {
        const float sum = lanes_sum(tail, min(sh.G, 64));
        float* const at = mine + t * len;
        auto add = [&]() {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (sh.lane + j * sh.G) * V;
                if (c < a.width) {
                    float o[V];
                    load_cols<V>(at + c, o);
#pragma unroll
                    for (int e = 0; e < V; ++e) o[e] += v[j][e];
                    store_cols<V>(at + c, o);
                }
                zero_cols<V>(v[j]);
            }
            if ((sh.lane & 63) == 0) at[len - kTail + (sh.G > 64 ? wave : 0)] += sum;
            tail = 0.f;
        };
        if (sh.G >= 64) {
            if (who) add();
            return;
        }
        const unsigned long long which = __ballot(who);
        for (int k = 0; k < 64; k += sh.G) {
            if (!((which >> k) & 1)) continue;
            if ((lane & ~(sh.G - 1)) == k) add();
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    int turn = 0, type = a.p.types ? -1 : 0;
    for (int64_t row0 = (int64_t)blockIdx.x * sh.rows_per_block; row0 < a.rows; row0 += (int64_t)gridDim.x * sh.rows_per_block) {
        const int64_t row = row0 + sh.group;
        const bool live = row < a.rows;
        const int t = row_type(a.p, row, live);
        const int64_t base = row * a.width;
        float x[NV][V], s[NV][V], dy[NV][V], dt[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (sh.lane + j * sh.G) * V;
            zero_cols<V>(x[j]);
            zero_cols<V>(s[j]);
            zero_cols<V>(dy[j]);
            zero_cols<V>(dt[j]);
            if (t >= 0 && c < a.width) {
                if constexpr (HELD) {
                    CodeWords<V> xw, sw;
                    load_codes<EVEN, V>(static_cast<const int8_t*>(a.a) + base, c, a.width, xw);
                    load_codes<EVEN, V>(static_cast<const int8_t*>(a.s) + base, c, a.width, sw);
                    const int64_t b = row * held_blocks(a.width) + c / kHeldBlock;
                    from_codes<V>(xw, held_step(a.a_scales[b]), x[j]);
                    from_codes<V>(sw, held_step(a.s_scales[b]), s[j]);
                } else {
                    load_v<EVEN>(static_cast<const TA*>(a.a) + base, c, a.width, x[j]);
                    load_v<EVEN>(static_cast<const TS*>(a.s) + base, c, a.width, s[j]);
                }
                if (a.dy) load_v<EVEN>(static_cast<const TO*>(a.dy) + base, c, a.width, dy[j]);
                if (a.ds) load_v<EVEN>(static_cast<const TS*>(a.ds) + base, c, a.width, dt[j]);
            }
        }
        const bool change = t >= 0 && t != type;
        if (__any(change)) {
            if (a.sums) give(change && type >= 0, max(type, 0), G, dscale);
            if (change) {
                type = t;
                scale = a.p.scale ? a.p.scale[t] : 1.f;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int c = (sh.lane + j * sh.G) * V;
                    if (a.p.gate && c < a.width) load_v<EVEN>(a.p.gate + (int64_t)t * a.width, c, a.width, gate[j]);
                }
            }
        }
        float none = 0.f, q1 = 1.f, k1 = 1.f;
        if (a.p.w1) {
            float sq = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) sq += dot_cols<V>(x[j], x[j]);
            row_sums(sq, none, sh.G, lds, turn++);
            if (!(sq <= FLT_MAX)) {          // as in the forward; the scaled values take their place
                k1 = kScaleDown;
                sq = 0.f;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        x[j][e] *= k1;
                        sq += x[j][e] * x[j][e];
                    }
                row_sums(sq, none, sh.G, lds, turn++);
            }
            q1 = rsqrtf(sq * inv + a.eps * k1 * k1);
        }
        if (a.dy) {
            float u[NV][V], sq = 0.f, gs = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    u[j][e] = scale * s[j][e] + gate[j][e] * (x[j][e] * q1 * w1[j][e]);
                    sq += u[j][e] * u[j][e];
                    gs += dy[j][e] * w2[j][e] * u[j][e];
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
            // (with v = k u: q(u) = k q(v), u q(u)^2 mean(g u) = v q(v)^2 mean(g v))
            const float q2 = rsqrtf(sq * inv + a.eps * k2 * k2), along = q2 * q2 * (gs * inv), qk = q2 * k2;
            if (t >= 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        dt[j][e] += qk * (dy[j][e] * w2[j][e] - u[j][e] * along);
                        dw2[j][e] += dy[j][e] * (u[j][e] * q2);
                    }
            }
        }
        float along = 0.f;
        if (a.p.w1) {
            float ha = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) ha += dt[j][e] * gate[j][e] * w1[j][e] * x[j][e];
            row_sums(ha, none, sh.G, lds, turn++);
            along = q1 * q1 * (ha * inv);
        }
        const float qk = q1 * k1;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (sh.lane + j * sh.G) * V;
            if (live && c < a.width && (t >= 0 || !a.accumulate)) {
                float da[V], dstream[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float h = dt[j][e] * gate[j][e] * w1[j][e];
                    da[e] = t >= 0 ? qk * (h - x[j][e] * along) : 0.f;
                    dstream[e] = t >= 0 ? scale * dt[j][e] : 0.f;
                    if (t >= 0) {
                        G[j][e] += dt[j][e] * (x[j][e] * q1);
                        dscale += dt[j][e] * s[j][e];
                    }
                }
                if (a.da) put<EVEN>(static_cast<TA*>(a.da) + base, c, a.width, da, a.accumulate);
                if (a.dstream) put<EVEN>(static_cast<TS*>(a.dstream) + base, c, a.width, dstream, a.accumulate);
            }
        }
    }
    if (!a.sums) return;
    give(type >= 0, max(type, 0), G, dscale);
    float unused = 0.f;
    give(true, T, dw2, unused);
    __syncthreads();
    for (int i = threadIdx.x; i < part_len(T, a.width); i += kBlock) {
        const int t = i / (a.width + 1), c = i - t * (a.width + 1);
        float v = 0.f;
        for (int k = 0; k < slots; ++k) {
            const float* const at = places + (k * (T + 1) + t) * len;
            if (c < a.width) {
                v += at[c];
            } else {
#pragma unroll
                for (int q = 0; q < kTail; ++q) v += at[len - kTail + q];
            }
        }
        if (gridDim.x > 1) a.part[(int64_t)blockIdx.x * part_len(T, a.width) + i] = v;
        else places[t * len + (c < a.width ? c : len - kTail)] = v;          // (no other lane reads these)
    }
    if (gridDim.x > 1) return;
    __syncthreads();
    for (int c = threadIdx.x; c <= a.width; c += kBlock) finish(a, c, [&](int t) { return places[t * len + (c < a.width ? c : len - kTail)]; });
}

// (what two turns of a workgroup finish is left to one: the sums then need no second launch)
inline int workgroups(const rgnn_block_norm_desc_t* d) {
    const JunctionPlan p = block_plan(d);
    return p.turns <= 2 ? (int)std::min<int64_t>(p.turns, 1) : (int)std::min<int64_t>(kMaxBlocks, p.turns);
}

template <typename TA, typename TS, typename TO, bool HELD>
rgnn_status_t launch_rows(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, const BlockBwdArgs& a, hipStream_t st) {
    return block_with_vectors<sizeof(TA) + sizeof(TS) + sizeof(TO) == 6>(d, p, [&](auto V, auto NV, auto even) -> rgnn_status_t {
        auto* const kernel = block_bwd_kernel<TA, TS, TO, V(), NV(), even(), HELD>;
        // (at most eight wavefronts' places of types * (width + 12) <= 4096: 160 KB)
        const size_t lds = sizeof(float) * (4 * kWaves + (a.sums ? (size_t)(p.G > 64 ? 1 : kWaves) * (d->types + 1) * place_len(d->width) : 0));
        RGNN_TRY(allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds));
        KernelTimer timer(st, "block_norm_bwd");
        kernel<<<workgroups(d), kBlock, lds, st>>>(a);
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
