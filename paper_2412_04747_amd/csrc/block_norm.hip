// The junction of a block's output with the residual stream (block_norm.h has the formulas): forward, and the entry points.
//
// Twelve operations per element against 8 to 16 bytes: the memory's rate is the bound.  A row's a and s stay in the registers of the lanes that loaded them from
// the first norm's sum to the second's, so that each tensor is passed once, where the two norms and the gate by themselves pass n and the sum again.
// The same registers are packed to 8 bits where the backward is to read them so.  Against 4.9 TB/s of a large copy: 1M rows of 64, fp32 to bf16, four types, 150 us (6.0 TB/s);
// 2M rows of 128, bf16, 364 (5.6); 200017 rows of 128, fp32, left in 8 bits too, 82 (5.6); one row 2.4.  Without norms, gate and scale of four mixed types, 1M rows of 64, fp32, 130 (5.9).
// Rows of odd widths are further off, with some lanes idle and rows at any address: 30011 of 349, fp32, 39 (4.3), seven mixed types 50 (3.4); bf16, by vectors of four columns too and so
// with fp32's instructions for half its bytes, 28 and 39 (3.0, 2.1).
#include <float.h>

#include "rgnn_internal.h"
#include "device_utils.h"
#include "block_norm.h"

namespace rgnn {

namespace {

// Workgroups of four wavefronts (of whole rows: eight): with the next row's tensors on their way, four to a compute unit are enough for 4 columns per lane, three for more.  In us,
// with 512 / 768 / 1024 / 1536:  1M rows of 64, fp32: 181 / 177 / 179 / 192; 500000 of mixed types: 101 / 97 / 89 / 90; 200017 of 128 left in 8 bits: 93 / 84 / 80 / 81
//                                2M rows of 128, bf16: 357 / 365 / 377 / 404; 500000: 90 / 87 / 88 / 94; 200000 rows of 349, fp32: 226 / 238 / 256 / 258
constexpr int most_blocks(int cols, int GC) { return cols <= 4 || GC == kBlock ? 1024 : 768; }
constexpr int kMaxWidth = 8192;

// Codes and scales of vector j of a row, by all its lanes; live: the row is one of the tensor's.
template <typename S>
__device__ __forceinline__ void pack_cols(const RowLanes<S>& sh, const float (&v)[S::V], int64_t row0, int j, bool live, int8_t* codes, uint8_t* scales) {
    constexpr int V = S::V;
    const unsigned b = scale_byte(lanes_max(bits_max(v), min(sh.G, kHeldBlock / V)));
    CodeWords<V> w;
    to_codes(v, b, w);
    if (!live || !sh.in(j)) return;
    const int c = sh.col(j), nb = held_blocks(sh.width);
    store_codes<S::LIE == kEven, V>(sh.template row<int8_t>(codes, row0), c, sh.width, w);
    if (c % kHeldBlock == 0) (scales + row0 * nb)[(unsigned)(sh.group * nb + c / kHeldBlock)] = (uint8_t)b;
}

template <typename TA, typename TS, typename TO, typename S>
__global__ __launch_bounds__(block_threads(S::GC)) void block_fwd_kernel(BlockFwdArgs a) {
    constexpr int V = S::V, NV = S::NV;
    constexpr bool EVEN = S::LIE == kEven;
    __shared__ float lds[4 * (kBlock / 64)];
    const RowLanes<S> sh(a.G, a.width);
    constexpr bool AHEAD = V * NV <= 8;
    const float inv = 1.f / (float)a.width;
    // gw: gate w1 of the type at hand
    float w2[NV][V], gw[NV][V], scale = 1.f;
    auto load_type = [&](int t) {
        scale = a.p.scale ? a.p.scale[t] : 1.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!sh.in(j)) continue;
            float w[V];
#pragma unroll
            for (int e = 0; e < V; ++e) gw[j][e] = w[e] = 1.f;
            if (a.p.gate) sh.shared(a.p.gate + (unsigned)(t * a.width), j, gw[j]);
            if (a.p.w1) sh.shared(a.p.w1, j, w);
#pragma unroll
            for (int e = 0; e < V; ++e) gw[j][e] *= w[e];
        }
    };
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        zero_cols<V>(gw[j]);
        zero_cols<V>(w2[j]);
        if (a.p.w2 && sh.in(j)) sh.shared(a.p.w2, j, w2[j]);
    }
    load_type(0);
    // A row's tensors as they lie in memory: the next row's are on their way while a row is worked on, and its type is known before.
    RawCols<TA, V> xr[NV];
    RawCols<TS, V> sr[NV];
    auto fetch = [&](int64_t row0, int t) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (t >= 0 && sh.in(j)) {
                sh.template fetch<TA>(a.a, row0, j, xr[j]);
                sh.template fetch<TS>(a.s, row0, j, sr[j]);
            } else {
#pragma unroll
                for (int k = 0; k < (int)(sizeof(xr[j]) / 4); ++k) xr[j][k] = 0;
#pragma unroll
                for (int k = 0; k < (int)(sizeof(sr[j]) / 4); ++k) sr[j][k] = 0;
            }
        }
    };
    const int64_t step = (int64_t)gridDim.x * sh.rows();
    int turn = 0, type = 0;
    int64_t row0 = (int64_t)blockIdx.x * sh.rows();
    int now = sh.type(a.p, row0, a.rows), next = sh.type(a.p, row0 + step, a.rows);
    if constexpr (AHEAD) fetch(row0, now);
    // (the trip count is the same for all threads of a workgroup whose rows are its own: the barrier in row_sum)
    for (; row0 < a.rows; row0 += step) {
        const int t = now;
        const bool live = row0 + sh.group < a.rows;
        if constexpr (!AHEAD) fetch(row0, t);
        float x[NV][V], s[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            sh.template values<TA>(j, xr[j], x[j]);
            sh.template values<TS>(j, sr[j], s[j]);
        }
        now = next;
        if constexpr (AHEAD) fetch(row0 + step, now);
        next = sh.type(a.p, row0 + 2 * step, a.rows);
        if (t >= 0 && t != type) {
            type = t;
            load_type(t);
        }
        if (a.a_codes) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                pack_cols(sh, x[j], row0, j, live, a.a_codes, a.a_scales);
                pack_cols(sh, s[j], row0, j, live, a.s_codes, a.s_scales);
            }
        }
        float q1 = 1.f, k1 = 1.f;
        if (a.p.w1) {
            float sq = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) sq += dot_cols<V>(x[j], x[j]);
            row_sum(sq, sh.G, lds, turn++);
            if (!(sq <= FLT_MAX)) {          // (all lanes of the row, and where the row is a workgroup's, all of it)
                k1 = kScaleDown;
                sq = 0.f;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) sq += (x[j][e] * k1) * (x[j][e] * k1);
                row_sum(sq, sh.G, lds, turn++);
            }
            q1 = rsqrtf(sq * inv + a.eps * k1 * k1);
        }
        float sq = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s[j][e] = scale * s[j][e] + x[j][e] * k1 * q1 * gw[j][e];
                sq += s[j][e] * s[j][e];
            }
        float q2 = 1.f, k2 = 1.f;
        if (a.out) {
            row_sum(sq, sh.G, lds, turn++);
            if (!(sq <= FLT_MAX)) {
                k2 = kScaleDown;
                sq = 0.f;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) sq += (s[j][e] * k2) * (s[j][e] * k2);
                row_sum(sq, sh.G, lds, turn++);
            }
            q2 = rsqrtf(sq * inv + a.eps * k2 * k2);
        }
        TS* const sum_row = sh.template row<TS>(a.sum, row0);
        TO* const out_row = sh.template row<TO>(a.out, row0);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!live || !sh.in(j)) continue;
            float y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s[j][e] = t >= 0 ? s[j][e] : 0.f;
                y[e] = t >= 0 ? s[j][e] * q2 * k2 * w2[j][e] : 0.f;
            }
            auto out = [&](auto* to, const float (&v)[V]) {
                if constexpr (EVEN)
                    if (a.streaming) return store_cols_nt<V>(to + sh.col(j), v);
                store_v<EVEN>(to, sh.col(j), a.width, v);
            };
            if (a.sum) out(sum_row, s[j]);
            if (a.out) out(out_row, y);
        }
    }
}

template <typename TA, typename TS, typename TO>
rgnn_status_t launch_fwd(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, const BlockFwdArgs& a, hipStream_t st) {
    return block_with_shape<sizeof(TA) + sizeof(TS) + sizeof(TO) == 6>(d, p, [&](auto shape) -> rgnn_status_t {
        using S = decltype(shape);
        KernelTimer timer(st, "block_norm_fwd");
        block_fwd_kernel<TA, TS, TO, S><<<(unsigned)std::min<int64_t>(most_blocks(S::V * S::NV, S::GC), p.turns), block_threads(S::GC), 0, st>>>(a);
        RGNN_CHECK_LAUNCH();
        return RGNN_OK;
    });
}

rgnn_status_t check_desc(const rgnn_block_norm_desc_t* d) {
    if (!d) RGNN_FAIL(RGNN_EINVAL, "desc is NULL");
    RGNN_TRY(check_rows(d->rows));
    if (d->width < 1) RGNN_FAIL(RGNN_EINVAL, "width %d is not positive", d->width);
    if (d->width > kMaxWidth) RGNN_FAIL(RGNN_EUNSUPPORTED, "width %d not supported (up to %d)", d->width, kMaxWidth);
    for (int32_t t : {d->a_dtype, d->sum_dtype, d->out_dtype}) RGNN_TRY(check_dtype(t));
    if (d->types < 1) RGNN_FAIL(RGNN_EINVAL, "types %d is not positive", d->types);
    if (!block_types_fit(d->types, d->width))
        RGNN_FAIL(RGNN_EUNSUPPORTED, "types %d of width %d not supported (types * (width + 12) up to 4096; up to 32 types of up to 1024 columns: (types + 1) * (width + 12) up to 9600)",
                  d->types, d->width);
    if (!(d->eps >= 0.f) || d->eps == INFINITY) RGNN_FAIL(RGNN_EINVAL, "eps is not a finite number >= 0");
    if (d->flags & ~RGNN_FLAG_ACCUMULATE) RGNN_FAIL(RGNN_EINVAL, "flags: only RGNN_FLAG_ACCUMULATE applies");
    return RGNN_OK;
}

// The parameters' memory, and whether they fit the descriptor.
struct ParamSpans { Span types, w1, gate, scale, w2; };
rgnn_status_t check_params(const rgnn_block_norm_desc_t* d, const rgnn_block_norm_params_t* p, ParamSpans& s) {
    if (!p) RGNN_FAIL(RGNN_EINVAL, "params is NULL");
    if (!p->row_types && d->types > 1 && d->rows > 0) RGNN_FAIL(RGNN_EINVAL, "row_types is NULL with %d types", d->types);
    const size_t n = (size_t)d->types * d->width;
    s = ParamSpans{Span{reinterpret_cast<const char*>(p->row_types), 4 * (size_t)d->rows}, span(p->w_after, d->width, RGNN_F32), span(p->gate, n, RGNN_F32),
                   span(p->scale, d->types, RGNN_F32), span(p->w_before, d->width, RGNN_F32)};
    for (const Span& q : {s.types, s.w1, s.gate, s.scale, s.w2}) RGNN_TRY(check_aligned(q));
    return RGNN_OK;
}
BlockParams device_params(const rgnn_block_norm_desc_t* d, const rgnn_block_norm_params_t* p) {
    return BlockParams{p->row_types, d->types, p->w_after, p->gate, p->scale, p->w_before};
}

rgnn_status_t check_held(const rgnn_rows8_t* a8, const rgnn_rows8_t* s8) {
    if (!a8 != !s8) RGNN_FAIL(RGNN_EINVAL, "a8 and s8 are given together or not at all");
    for (const rgnn_rows8_t* r : {a8, s8})
        if (r && (!r->codes || !r->scales)) RGNN_FAIL(RGNN_EINVAL, "codes or scales of a8 or s8 is NULL");
    return RGNN_OK;
}

}  // namespace

}  // namespace rgnn

using namespace rgnn;

extern "C" rgnn_status_t rgnn_block_norm_workspace_bytes(const rgnn_block_norm_desc_t* desc, size_t* bwd_workspace) {
    RGNN_TRY(check_desc(desc));
    if (!bwd_workspace) RGNN_FAIL(RGNN_EINVAL, "bwd_workspace is NULL");
    *bwd_workspace = block_bwd_workspace(desc);
    return RGNN_OK;
}

extern "C" rgnn_status_t rgnn_block_norm_fwd(const rgnn_block_norm_desc_t* desc, const rgnn_block_norm_params_t* params, const void* a, const void* s, void* sum,
                                             void* out, const rgnn_rows8_t* a8, const rgnn_rows8_t* s8, void* stream) {
    RGNN_TRY(check_desc(desc));
    ParamSpans ps;
    RGNN_TRY(check_params(desc, params, ps));
    if (desc->rows == 0) return RGNN_OK;
    if (!a || !s) RGNN_FAIL(RGNN_EINVAL, "a or s is NULL");
    if (!out != !params->w_before) RGNN_FAIL(RGNN_EINVAL, "out and w_before are given together or not at all");
    RGNN_TRY(check_held(a8, s8));
    if (!sum && !out && !a8) RGNN_FAIL(RGNN_EINVAL, "no result is wanted: sum, out and a8 are NULL");
    const int64_t rows = desc->rows;
    const int width = desc->width;
    const size_t n = (size_t)rows * width;
    const Span as = span(a, n, desc->a_dtype), ss = span(s, n, desc->sum_dtype), sums = span(sum, n, desc->sum_dtype), outs = span(out, n, desc->out_dtype);
    Span held[4] = {};
    if (a8) held[0] = code_span(a8, rows, width), held[1] = scale_span(a8, rows, width), held[2] = code_span(s8, rows, width), held[3] = scale_span(s8, rows, width);
    for (const Span& q : {as, ss, sums, outs, held[0], held[2]}) RGNN_TRY(check_aligned(q));
    for (const Span& o : {sums, outs, held[0], held[1], held[2], held[3]})
        for (const Span& q : {ps.types, ps.w1, ps.gate, ps.scale, ps.w2})
            if (o.overlaps(q)) RGNN_FAIL(RGNN_EINVAL, "a result overlaps a parameter");
    // a row's lanes have read it before they write it: in place is fine, a shifted overlap is not
    for (const Span& o : {sums, outs})
        if ((o.overlaps(as) && !o.same(as)) || (o.overlaps(ss) && !o.same(ss)))
            RGNN_FAIL(RGNN_EINVAL, "sum or out overlaps an input that it is not the buffer of");
    if (sums.overlaps(outs)) RGNN_FAIL(RGNN_EINVAL, "sum and out overlap");
    for (int i = 0; i < 4; ++i) {
        for (const Span& q : {as, ss, sums, outs})
            if (held[i].overlaps(q)) RGNN_FAIL(RGNN_EINVAL, "a8 or s8 overlaps a tensor");
        for (int j = 0; j < i; ++j)
            if (held[i].overlaps(held[j])) RGNN_FAIL(RGNN_EINVAL, "codes and scales of a8 and s8 overlap");
    }
    const JunctionPlan p = block_plan(desc);
    BlockFwdArgs f{rows, width, p.G, (int64_t)(sums.bytes + outs.bytes) > kCachedBytes, desc->eps, device_params(desc, params), a, s, sum, out, nullptr, nullptr, nullptr, nullptr};
    if (a8) f.a_codes = a8->codes, f.a_scales = a8->scales, f.s_codes = s8->codes, f.s_scales = s8->scales;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return block_with_types(desc, [&](auto ta, auto ts, auto to) { return launch_fwd<decltype(ta), decltype(ts), decltype(to)>(desc, p, f, st); });
}

extern "C" rgnn_status_t rgnn_block_norm_bwd(const rgnn_block_norm_desc_t* desc, const rgnn_block_norm_params_t* params, const void* a, const void* s,
                                             const rgnn_rows8_t* a8, const rgnn_rows8_t* s8, const void* dOut, const void* dSum, void* dA, void* dS,
                                             const rgnn_block_norm_grads_t* grads, void* workspace, void* stream) {
    RGNN_TRY(check_desc(desc));
    ParamSpans ps;
    RGNN_TRY(check_params(desc, params, ps));
    const rgnn_block_norm_grads_t g = grads ? *grads : rgnn_block_norm_grads_t{};
    if ((g.w_after && !params->w_after) || (g.gate && !params->gate) || (g.scale && !params->scale) || (g.w_before && !params->w_before))
        RGNN_FAIL(RGNN_EINVAL, "the gradient of a parameter that is not given");
    const bool sums = g.w_after || g.gate || g.scale || g.w_before;
    if (sums && !workspace) RGNN_FAIL(RGNN_EWORKSPACE, "workspace is NULL");
    const Span gs[4] = {span(g.w_after, desc->width, RGNN_F32), span(g.gate, (size_t)desc->types * desc->width, RGNN_F32), span(g.scale, desc->types, RGNN_F32),
                        span(g.w_before, desc->width, RGNN_F32)};
    const Span work{sums ? static_cast<const char*>(workspace) : nullptr, block_bwd_workspace(desc)};
    for (const Span& q : {gs[0], gs[1], gs[2], gs[3], work}) RGNN_TRY(check_aligned(q));
    const bool held = a8 || s8;
    Span in[6] = {}, das{}, dss{};
    if (desc->rows > 0) {
        RGNN_TRY(check_held(a8, s8));
        if (held ? a || s : !a || !s) RGNN_FAIL(RGNN_EINVAL, "a and s are given, or a8 and s8 are, and the others are NULL");
        if (dOut && !params->w_before) RGNN_FAIL(RGNN_EINVAL, "dOut is given, w_before is NULL");
        if (!dOut && !dSum) RGNN_FAIL(RGNN_EINVAL, "dOut and dSum are both NULL");
        const int64_t rows = desc->rows;
        const int width = desc->width;
        const size_t n = (size_t)rows * width;
        in[0] = held ? code_span(a8, rows, width) : span(a, n, desc->a_dtype);
        in[1] = held ? code_span(s8, rows, width) : span(s, n, desc->sum_dtype);
        in[2] = span(dOut, n, desc->out_dtype);
        in[3] = span(dSum, n, desc->sum_dtype);
        if (held) in[4] = scale_span(a8, rows, width), in[5] = scale_span(s8, rows, width);
        das = span(dA, n, desc->a_dtype);
        dss = span(dS, n, desc->sum_dtype);
        for (const Span& q : {in[0], in[1], in[2], in[3], das, dss}) RGNN_TRY(check_aligned(q));
        for (const Span& o : {das, dss})
            for (int i = 0; i < 6; ++i)
                if (o.overlaps(in[i]) && !((i == 2 || i == 3) && o.same(in[i]))) RGNN_FAIL(RGNN_EINVAL, "dA or dS overlaps a tensor that it is not the buffer of");
        if (das.overlaps(dss)) RGNN_FAIL(RGNN_EINVAL, "dA and dS overlap");
    }
    for (const Span& o : {das, dss, gs[0], gs[1], gs[2], gs[3], work})
        for (const Span& q : {ps.types, ps.w1, ps.gate, ps.scale, ps.w2})
            if (o.overlaps(q)) RGNN_FAIL(RGNN_EINVAL, "a result or the workspace overlaps a parameter");
    const Span small[5] = {gs[0], gs[1], gs[2], gs[3], work};
    for (int i = 0; i < 5; ++i) {
        for (const Span& q : {in[0], in[1], in[2], in[3], in[4], in[5], das, dss})
            if (small[i].overlaps(q)) RGNN_FAIL(RGNN_EINVAL, "a parameter's gradient or the workspace overlaps a tensor");
        for (int j = 0; j < i; ++j)
            if (small[i].overlaps(small[j])) RGNN_FAIL(RGNN_EINVAL, "two parameters' gradients, or one and the workspace, overlap");
    }
    const int accumulate = (desc->flags & RGNN_FLAG_ACCUMULATE) != 0;
    BlockBwdArgs b{desc->rows, desc->width, block_plan(desc).G, accumulate, !accumulate && (int64_t)(das.bytes + dss.bytes) > kCachedBytes, desc->eps, device_params(desc, params), a, s,
                   nullptr, nullptr, dOut, dSum, dA, dS, sums, nullptr, g};
    if (held && desc->rows > 0) b.a = a8->codes, b.a_scales = a8->scales, b.s = s8->codes, b.s_scales = s8->scales;
    return block_bwd(desc, b, held, workspace, static_cast<hipStream_t>(stream));
}
