// The entry points around a unit (include/rtp.h): argument checks, and the calls that launch the kernels.  Nothing reaches
// the runtime before every check has passed.
#include "rtp_block_kernels.h"
#include "rtp_error.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

using namespace rtp;

static bool dtype_ok(rtp_dtype t) { return t == RTP_F32 || t == RTP_BF16 || t == RTP_F16; }
static size_t esize(rtp_dtype t) { return t == RTP_F32 ? 4 : 2; }
static bool aligned(const void *p, size_t to) { return (uintptr_t)p % to == 0; }
constexpr int64_t MAX_T = (int64_t)1 << 31, MAX_LD = (int64_t)1 << 28; // offsets stay within 64 bits

// a leading dimension: 0 stands for the row length
static bool take_ld(int64_t &ld, int64_t cols)
{
    if (ld == 0) ld = cols;
    return ld >= cols && ld <= MAX_LD;
}

// ---------------------------------------------------------------------------
// router
// ---------------------------------------------------------------------------
static rtp_status route_check(const char *who, rtp_route_desc &d)
{
    if (!dtype_ok(d.dtype) || (d.score != RTP_SCORE_SOFTMAX && d.score != RTP_SCORE_SIGMOID))
        return fail(RTP_ERR_INVALID, "%s: bad dtype or score", who);
    if (!std::isfinite(d.scale)) return fail(RTP_ERR_INVALID, "%s: the scale is not finite", who);
    if (d.T < 0 || d.T > MAX_T || d.E < 1 || d.k < 1 || d.groups < 1 || d.kept_groups < 1 || d.kept_groups > d.groups)
        return fail(RTP_ERR_SHAPE, "%s: T=%lld E=%d k=%d groups=%d kept_groups=%d", who, (long long)d.T, d.E, d.k, d.groups, d.kept_groups);
    if (d.E > RTP_ROUTE_MAX_EXPERTS || d.k > RTP_ROUTE_MAX_TOP || d.groups > RTP_ROUTE_MAX_GROUPS)
        return fail(RTP_ERR_UNSUPPORTED, "%s: at most %d experts, %d choices, %d groups", who, RTP_ROUTE_MAX_EXPERTS, RTP_ROUTE_MAX_TOP,
                    RTP_ROUTE_MAX_GROUPS);
    if (d.E % d.groups) return fail(RTP_ERR_SHAPE, "%s: %d groups do not divide %d experts", who, d.groups, d.E);
    if (d.k > d.E / d.groups * d.kept_groups) return fail(RTP_ERR_SHAPE, "%s: %d choices out of %d eligible experts", who, d.k, d.E / d.groups * d.kept_groups);
    if (d.group_top != 1 && d.group_top != 2) return fail(RTP_ERR_INVALID, "%s: group_top is 1 or 2", who);
    if (!take_ld(d.ld, d.E) || !take_ld(d.ld_grad, d.E)) return fail(RTP_ERR_SHAPE, "%s: bad leading dimension", who);
    return RTP_OK;
}

extern "C" rtp_status rtp_route_fwd(const rtp_route_desc *desc, const void *logits, const float *bias, int32_t *ids, float *weights, void *stream)
{
    const char *who = "rtp_route_fwd";
    if (!desc) return fail(RTP_ERR_INVALID, "%s: null argument", who);
    rtp_route_desc d = *desc;
    RTP_TRY(route_check(who, d));
    if (d.T == 0) return RTP_OK;
    if (!logits || !ids || !weights) return fail(RTP_ERR_INVALID, "%s: null pointer", who);
    if (!aligned(logits, esize(d.dtype)) || !aligned(bias, 4) || !aligned(ids, 4) || !aligned(weights, 4))
        return fail(RTP_ERR_SHAPE, "%s: pointers must be multiples of the element size", who);
    HIP_TRY(launch_route_fwd(d, logits, bias, ids, weights, (hipStream_t)stream));
    return RTP_OK;
}

extern "C" rtp_status rtp_route_bwd(const rtp_route_desc *desc, const void *logits, const int32_t *ids, const float *dweights, void *dlogits,
                                    void *stream)
{
    const char *who = "rtp_route_bwd";
    if (!desc) return fail(RTP_ERR_INVALID, "%s: null argument", who);
    rtp_route_desc d = *desc;
    RTP_TRY(route_check(who, d));
    if (!dtype_ok(d.grad_dtype)) return fail(RTP_ERR_INVALID, "%s: bad gradient dtype", who);
    if (d.T == 0) return RTP_OK;
    if (!logits || !ids || !dweights || !dlogits) return fail(RTP_ERR_INVALID, "%s: null pointer", who);
    if (logits == dlogits) return fail(RTP_ERR_INVALID, "%s: the gradient overlaps the logits", who);
    if (!aligned(logits, esize(d.dtype)) || !aligned(dlogits, esize(d.grad_dtype)) || !aligned(ids, 4) || !aligned(dweights, 4))
        return fail(RTP_ERR_SHAPE, "%s: pointers must be multiples of the element size", who);
    HIP_TRY(launch_route_bwd(d, logits, ids, dweights, dlogits, (hipStream_t)stream));
    return RTP_OK;
}

// ---------------------------------------------------------------------------
// combination
// ---------------------------------------------------------------------------
static rtp_status combine_check(const char *who, CombineArgs &a)
{
    if (!dtype_ok(a.dtype)) return fail(RTP_ERR_INVALID, "%s: bad dtype", who);
    if (a.T < 0 || a.k < 1 || a.T > MAX_T / a.k || a.D < 1 || a.D > RTP_COMBINE_MAX_D)
        return fail(RTP_ERR_SHAPE, "%s: T=%lld k=%d D=%lld", who, (long long)a.T, a.k, (long long)a.D);
    if (a.k > RTP_COMBINE_MAX_TOP) return fail(RTP_ERR_UNSUPPORTED, "%s: at most %d slots a token", who, RTP_COMBINE_MAX_TOP);
    if (!take_ld(a.ld_y, a.D) || !take_ld(a.ld_yk, a.D) || !take_ld(a.ld_dyk, a.D)) return fail(RTP_ERR_SHAPE, "%s: bad leading dimension", who);
    const size_t es = esize(a.dtype);
    for (const void *p : {a.dY, a.Yk, (const void *)a.Y, (const void *)a.dYk})
        if (!aligned(p, es)) return fail(RTP_ERR_SHAPE, "%s: pointers must be multiples of the element size", who);
    if (!aligned(a.weights, 4) || !aligned(a.dweights, 4)) return fail(RTP_ERR_SHAPE, "%s: pointers must be multiples of the element size", who);
    return RTP_OK;
}

extern "C" rtp_status rtp_combine_fwd(int64_t T, int k, int64_t D, rtp_dtype dtype, const void *Yk, int64_t ld_yk, const float *weights, void *Y,
                                      int64_t ld_y, void *stream)
{
    const char *who = "rtp_combine_fwd";
    CombineArgs a{};
    a.T = T; a.k = k; a.D = D; a.dtype = dtype;
    a.Yk = Yk; a.ld_yk = ld_yk; a.weights = weights; a.Y = Y; a.ld_y = ld_y;
    RTP_TRY(combine_check(who, a));
    if (T == 0) return RTP_OK;
    if (!Yk || !Y) return fail(RTP_ERR_INVALID, "%s: null pointer", who);
    if (Yk == Y) return fail(RTP_ERR_INVALID, "%s: the output overlaps the input", who);
    HIP_TRY(launch_combine_fwd(a, (hipStream_t)stream));
    return RTP_OK;
}

extern "C" rtp_status rtp_combine_bwd(int64_t T, int k, int64_t D, rtp_dtype dtype, const void *dY, int64_t ld_dy, const void *Yk, int64_t ld_yk,
                                      const float *weights, void *dYk, int64_t ld_dyk, float *dweights, void *stream)
{
    const char *who = "rtp_combine_bwd";
    CombineArgs a{};
    a.T = T; a.k = k; a.D = D; a.dtype = dtype;
    a.dY = dY; a.ld_y = ld_dy; a.Yk = Yk; a.ld_yk = ld_yk; a.weights = weights; a.dYk = dYk; a.ld_dyk = ld_dyk; a.dweights = dweights;
    RTP_TRY(combine_check(who, a));
    if (T == 0 || (!dYk && !dweights)) return RTP_OK;
    if (!dY || (dweights && !Yk)) return fail(RTP_ERR_INVALID, "%s: null pointer", who);
    if (dYk && (dYk == dY || dYk == Yk)) return fail(RTP_ERR_INVALID, "%s: the output overlaps an input", who);
    HIP_TRY(launch_combine_bwd(a, (hipStream_t)stream));
    return RTP_OK;
}

// ---------------------------------------------------------------------------
// norms
// ---------------------------------------------------------------------------
static rtp_status norm_check(const char *who, rtp_norm_desc &d)
{
    if ((d.kind != RTP_NORM_RMS && d.kind != RTP_NORM_LAYER) || !dtype_ok(d.dtype) || !dtype_ok(d.stream_dtype))
        return fail(RTP_ERR_INVALID, "%s: bad kind or dtype", who);
    if (d.stream_dtype != d.dtype && d.stream_dtype != RTP_F32)
        return fail(RTP_ERR_UNSUPPORTED, "%s: the stream is of the units' dtype or fp32", who);
    const unsigned all = RTP_NORM_JOIN | RTP_NORM_POST | RTP_NORM_PRE;
    if ((d.parts & ~all) || !(d.parts & (RTP_NORM_JOIN | RTP_NORM_PRE)) || ((d.parts & RTP_NORM_POST) && !(d.parts & RTP_NORM_JOIN)))
        return fail(RTP_ERR_INVALID, "%s: bad parts %u", who, d.parts);
    if (d.gate != RTP_GATE_NONE && d.gate != RTP_GATE_CHANNEL && d.gate != RTP_GATE_ELEMENT) return fail(RTP_ERR_INVALID, "%s: bad gate", who);
    if (d.gate != RTP_GATE_NONE && !(d.parts & RTP_NORM_JOIN)) return fail(RTP_ERR_INVALID, "%s: a gate without a branch", who);
    if (d.T < 0 || d.T > MAX_T || d.D < 1 || d.D > RTP_NORM_MAX_D)
        return fail(RTP_ERR_SHAPE, "%s: T=%lld D=%lld", who, (long long)d.T, (long long)d.D);
    if (!(d.eps > 0.0f) || !std::isfinite(d.eps) || !std::isfinite(d.res_scale) || !std::isfinite(d.out_scale))
        return fail(RTP_ERR_INVALID, "%s: eps must be positive, the scales finite", who);
    if (!(d.parts & RTP_NORM_POST)) d.w_post_dev = d.b_post_dev = nullptr;
    if (!(d.parts & RTP_NORM_PRE)) d.w_pre_dev = d.b_pre_dev = nullptr;
    if (d.gate == RTP_GATE_NONE) d.gate_dev = nullptr;
    if (!take_ld(d.ld_gate, d.D)) return fail(RTP_ERR_SHAPE, "%s: bad leading dimension", who);
    return RTP_OK;
}

// the pointers of a call: what they must be multiples of
static rtp_status norm_pointers(const char *who, const rtp_norm_desc &d, std::initializer_list<const void *> stream, std::initializer_list<const void *> unit,
                                std::initializer_list<const void *> f32)
{
    bool ok = aligned(d.gate_dev, d.gate == RTP_GATE_ELEMENT ? esize(d.dtype) : 4);
    for (const void *p : stream) ok &= aligned(p, esize(d.stream_dtype));
    for (const void *p : unit) ok &= aligned(p, esize(d.dtype));
    for (const void *p : f32) ok &= aligned(p, 4);
    for (const float *p : {d.w_post_dev, d.b_post_dev, d.w_pre_dev, d.b_pre_dev}) ok &= aligned(p, 4);
    return ok ? RTP_OK : fail(RTP_ERR_SHAPE, "%s: pointers must be multiples of the element size", who);
}

extern "C" rtp_status rtp_norm_fwd(const rtp_norm_desc *desc, const rtp_norm_io *args, void *stream)
{
    const char *who = "rtp_norm_fwd";
    if (!desc || !args) return fail(RTP_ERR_INVALID, "%s: null argument", who);
    rtp_norm_desc d = *desc;
    rtp_norm_io io = *args;
    RTP_TRY(norm_check(who, d));
    const bool join = d.parts & RTP_NORM_JOIN, pre = d.parts & RTP_NORM_PRE;
    if (!join) { io.y_dev = nullptr; io.r_dev = nullptr; }
    if (!pre) io.h_dev = nullptr;
    if (!take_ld(io.ld_x, d.D) || !take_ld(io.ld_y, d.D) || !take_ld(io.ld_r, d.D) || !take_ld(io.ld_h, d.D))
        return fail(RTP_ERR_SHAPE, "%s: bad leading dimension", who);
    if (d.T == 0) return RTP_OK;
    const bool stats = pre || (d.parts & RTP_NORM_POST);
    if (!io.x_dev || (join && (!io.y_dev || !io.r_dev)) || (pre && !io.h_dev) || (stats && !io.stats_dev) || (d.gate != RTP_GATE_NONE && !d.gate_dev))
        return fail(RTP_ERR_INVALID, "%s: null pointer", who);
    if ((join && (io.r_dev == io.y_dev || (pre && io.r_dev == io.h_dev) || (io.r_dev == io.x_dev && io.ld_r != io.ld_x))) ||
        (pre && (io.h_dev == io.x_dev || (join && io.h_dev == io.y_dev))))
        return fail(RTP_ERR_INVALID, "%s: an output overlaps an input", who);
    RTP_TRY(norm_pointers(who, d, {io.x_dev, io.r_dev}, {io.y_dev, io.h_dev}, {io.stats_dev}));
    HIP_TRY(launch_norm_fwd(d, io, (hipStream_t)stream));
    return RTP_OK;
}

// the most column sums a description can ask for
static unsigned norm_sums(const rtp_norm_desc &d, bool w_pre, bool b_pre, bool w_post, bool b_post, bool gate)
{
    unsigned s = 0;
    gate = gate && d.gate == RTP_GATE_CHANNEL;
    if (d.parts & RTP_NORM_PRE) s |= (w_pre ? SUM_PRE_W : 0) | (b_pre ? SUM_PRE_B : 0);
    if (d.parts & RTP_NORM_POST) s |= (w_post ? SUM_POST_W : 0) | (b_post || (gate && d.b_post_dev) ? SUM_POST_B : 0);
    if (gate) s |= SUM_POST_W;
    return s;
}

extern "C" size_t rtp_norm_ws_bytes(const rtp_norm_desc *desc)
{
    if (!desc) return 0;
    rtp_norm_desc d = *desc;
    if (norm_check("rtp_norm_ws_bytes", d) != RTP_OK) return 0;
    return std::max<size_t>(16, (size_t)norm_bwd_parts(d) * __builtin_popcount(norm_sums(d, true, true, true, true, true)) * d.D * 4);
}

extern "C" rtp_status rtp_norm_bwd(const rtp_norm_desc *desc, const rtp_norm_grads *args, void *stream)
{
    const char *who = "rtp_norm_bwd";
    if (!desc || !args) return fail(RTP_ERR_INVALID, "%s: null argument", who);
    rtp_norm_desc d = *desc;
    rtp_norm_grads g = *args;
    RTP_TRY(norm_check(who, d));
    const bool join = d.parts & RTP_NORM_JOIN, pre = d.parts & RTP_NORM_PRE, post = d.parts & RTP_NORM_POST;
    const bool uses_y = post || d.gate != RTP_GATE_NONE;
    if (!uses_y) g.y_dev = nullptr;
    if (!join) g.dy_dev = nullptr;
    if (!pre) { g.r_dev = g.dh_dev = nullptr; g.dw_pre_dev = g.db_pre_dev = nullptr; }
    if (!post) g.dw_post_dev = g.db_post_dev = nullptr;
    if (d.gate == RTP_GATE_NONE) g.dgate_dev = nullptr;
    for (int64_t *ld : {&g.ld_r, &g.ld_y, &g.ld_dr, &g.ld_dh, &g.ld_dx, &g.ld_dy, &g.ld_dgate})
        if (!take_ld(*ld, d.D)) return fail(RTP_ERR_SHAPE, "%s: bad leading dimension", who);
    const bool stats = pre || post;
    const unsigned sums = norm_sums(d, g.dw_pre_dev, g.db_pre_dev, g.dw_post_dev, g.db_post_dev, g.dgate_dev);
    if (d.T == 0 && (!sums || g.accumulate)) return RTP_OK;
    if (d.T > 0) {
        if (!g.dx_dev || (join && !g.dy_dev) || (uses_y && !g.y_dev) || (pre && (!g.r_dev || !g.dh_dev)) || (stats && !g.stats_dev) ||
            (d.gate != RTP_GATE_NONE && !d.gate_dev) || (!pre && !g.dr_dev))
            return fail(RTP_ERR_INVALID, "%s: null pointer", who);
        if (g.dx_dev == g.r_dev || (g.dx_dev == g.dr_dev && g.ld_dx != g.ld_dr) || g.dx_dev == g.y_dev || g.dx_dev == g.dh_dev || g.dx_dev == g.dy_dev ||
            (join && (g.dy_dev == g.r_dev || g.dy_dev == g.y_dev || g.dy_dev == g.dr_dev || g.dy_dev == g.dh_dev)) ||
            (g.dgate_dev && (g.dgate_dev == d.gate_dev || g.dgate_dev == g.dx_dev || g.dgate_dev == g.dy_dev)))
            return fail(RTP_ERR_INVALID, "%s: an output overlaps an input", who);
    } else if (d.gate == RTP_GATE_CHANNEL && !d.gate_dev) {
        return fail(RTP_ERR_INVALID, "%s: null pointer", who);
    }
    if (sums && d.T > 0 && (!g.ws_dev || !aligned(g.ws_dev, 16))) return fail(RTP_ERR_INVALID, "%s: the workspace is missing or not a multiple of 16 bytes", who);
    if (sums && d.T > 0 && g.ws_bytes < (size_t)norm_bwd_parts(d) * __builtin_popcount(sums) * d.D * 4)
        return fail(RTP_ERR_SHAPE, "%s: the workspace is too small", who);
    RTP_TRY(norm_pointers(who, d, {g.r_dev, g.dr_dev, g.dx_dev}, {g.y_dev, g.dh_dev, g.dy_dev},
                          {g.stats_dev, g.dw_post_dev, g.db_post_dev, g.dw_pre_dev, g.db_pre_dev}));
    if (!aligned(g.dgate_dev, d.gate == RTP_GATE_ELEMENT ? esize(d.dtype) : 4)) return fail(RTP_ERR_SHAPE, "%s: pointers must be multiples of the element size", who);
    HIP_TRY(launch_norm_bwd(d, g, sums, (hipStream_t)stream));
    return RTP_OK;
}

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
struct rtp_adamw {
    rtp_moments moments;
    void *m, *v;
    uint8_t *exps;
    const AdamwEntry *entries;
    const int32_t *owner;
    int64_t chunks, blocks;
};

static bool adamw_sizes(const rtp_adamw_tensor *t, int count, int64_t *blocks, int64_t *chunks)
{
    if (!t || count < 1 || count > 1 << 20) return false;
    *blocks = *chunks = 0;
    for (int i = 0; i < count; ++i) {
        if (t[i].numel < 1 || t[i].numel > ((int64_t)1 << 40)) return false;
        *blocks += (t[i].numel + RTP_ADAMW_BLOCK - 1) / RTP_ADAMW_BLOCK;
        *chunks += (t[i].numel + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
        if (*blocks > (int64_t)1 << 26) return false; // (a grid of a workgroup for eight of them: 2^32 threads at 2^27)
    }
    return true;
}

extern "C" int64_t rtp_adamw_blocks(const rtp_adamw_tensor *t, int count)
{
    int64_t blocks, chunks;
    return adamw_sizes(t, count, &blocks, &chunks) ? blocks : -1;
}

extern "C" size_t rtp_adamw_table_bytes(const rtp_adamw_tensor *t, int count)
{
    int64_t blocks, chunks;
    return adamw_sizes(t, count, &blocks, &chunks) ? (size_t)count * sizeof(AdamwEntry) + (size_t)chunks * sizeof(int32_t) : 0;
}

// whether memory that a step writes overlaps other memory of it
static bool adamw_overlaps(const rtp_adamw_desc &d, int64_t blocks, size_t table_bytes)
{
    struct Span { uintptr_t from, to; bool written; };
    std::vector<Span> spans;
    spans.reserve((size_t)d.count * 3 + 4);
    auto add = [&](const void *p, size_t bytes, bool written) {
        if (p) spans.push_back({(uintptr_t)p, (uintptr_t)p + bytes, written});
    };
    for (int i = 0; i < d.count; ++i) {
        const rtp_adamw_tensor &t = d.tensors[i];
        add(t.param_dev, (size_t)t.numel * esize(t.dtype), true);
        add(t.master_dev, (size_t)t.numel * 4, true);
        add(t.grad_dev, (size_t)t.numel * 4, false);
    }
    const size_t each = d.moments == RTP_MOMENTS_F32 ? 4 : 1;
    add(d.m_dev, (size_t)blocks * RTP_ADAMW_BLOCK * each, true);
    add(d.v_dev, (size_t)blocks * RTP_ADAMW_BLOCK * each, true);
    if (d.moments == RTP_MOMENTS_8BIT) add(d.exps_dev, (size_t)blocks * 2, true);
    add(d.table_dev, table_bytes, true);
    std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.from < b.from; });
    uintptr_t end = 0, written_end = 0; // of what began earlier
    for (const Span &s : spans) {
        if (s.from < written_end || (s.written && s.from < end)) return true;
        end = std::max(end, s.to);
        if (s.written) written_end = std::max(written_end, s.to);
    }
    return false;
}

extern "C" rtp_status rtp_adamw_create(rtp_adamw **out, const rtp_adamw_desc *d)
{
    const char *who = "rtp_adamw_create";
    if (!out || !d) return fail(RTP_ERR_INVALID, "%s: null argument", who);
    *out = nullptr;
    if (d->moments != RTP_MOMENTS_F32 && d->moments != RTP_MOMENTS_8BIT) return fail(RTP_ERR_INVALID, "%s: bad kind of moments", who);
    int64_t blocks = 0, chunks = 0;
    if (!adamw_sizes(d->tensors, d->count, &blocks, &chunks)) return fail(RTP_ERR_SHAPE, "%s: no tensors, too many, or an empty one", who);
    if (!d->m_dev || !d->v_dev || !d->table_dev || (d->moments == RTP_MOMENTS_8BIT && !d->exps_dev)) return fail(RTP_ERR_INVALID, "%s: null pointer", who);
    if (!aligned(d->m_dev, 16) || !aligned(d->v_dev, 16) || !aligned(d->table_dev, 16) || (d->moments == RTP_MOMENTS_8BIT && !aligned(d->exps_dev, 2)))
        return fail(RTP_ERR_SHAPE, "%s: moments and table must be multiples of 16 bytes, exponents of 2", who);
    for (int i = 0; i < d->count; ++i) {
        const rtp_adamw_tensor &t = d->tensors[i];
        if (!dtype_ok(t.dtype)) return fail(RTP_ERR_INVALID, "%s: tensor %d: bad dtype", who, i);
        if (!t.param_dev || !t.grad_dev) return fail(RTP_ERR_INVALID, "%s: tensor %d: null pointer", who, i);
        if (t.dtype == RTP_F32 && t.master_dev) return fail(RTP_ERR_INVALID, "%s: tensor %d: an fp32 parameter has no master copy", who, i);
        if (!std::isfinite(t.weight_decay)) return fail(RTP_ERR_INVALID, "%s: tensor %d: the weight decay is not finite", who, i);
        if (!aligned(t.param_dev, esize(t.dtype)) || !aligned(t.grad_dev, 4) || !aligned(t.master_dev, 4))
            return fail(RTP_ERR_SHAPE, "%s: tensor %d: pointers must be multiples of the element size", who, i);
    }
    const size_t bytes = rtp_adamw_table_bytes(d->tensors, d->count);
    rtp_adamw *o = nullptr;
    std::vector<char> table;
    try {
        if (adamw_overlaps(*d, blocks, bytes)) return fail(RTP_ERR_INVALID, "%s: memory that a step writes overlaps other memory of it", who);
        table.resize(bytes);
        o = new rtp_adamw;
    } catch (const std::bad_alloc &) {
        return fail(RTP_ERR_INVALID, "%s: out of host memory", who);
    }
    *o = {d->moments, d->m_dev, d->v_dev, d->exps_dev, (const AdamwEntry *)d->table_dev,
          (const int32_t *)((const char *)d->table_dev + (size_t)d->count * sizeof(AdamwEntry)), chunks, blocks};
    AdamwEntry *e = (AdamwEntry *)table.data();
    int32_t *owner = (int32_t *)(table.data() + (size_t)d->count * sizeof(AdamwEntry));
    int64_t block = 0, chunk = 0;
    for (int i = 0; i < d->count; ++i) {
        const rtp_adamw_tensor &t = d->tensors[i];
        e[i] = {t.param_dev, t.grad_dev, t.master_dev, t.numel, block, chunk, (int)t.dtype, t.weight_decay};
        const int64_t n = (t.numel + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
        std::fill(owner + chunk, owner + chunk + n, i);
        block += (t.numel + RTP_ADAMW_BLOCK - 1) / RTP_ADAMW_BLOCK;
        chunk += n;
    }
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    hipError_t err = hipStreamIsCapturing((hipStream_t)d->stream, &cap);
    if (err == hipSuccess && cap != hipStreamCaptureStatusNone) {
        delete o;
        return fail(RTP_ERR_UNSUPPORTED, "%s: the stream is being captured into a graph", who);
    }
    if (err == hipSuccess) err = hipMemcpyAsync(d->table_dev, table.data(), bytes, hipMemcpyHostToDevice, (hipStream_t)d->stream);
    if (err == hipSuccess) err = hipStreamSynchronize((hipStream_t)d->stream);
    if (err != hipSuccess) {
        delete o;
        return fail(RTP_ERR_HIP, "%s: %s", who, hipGetErrorString(err));
    }
    *out = o;
    return RTP_OK;
}

extern "C" rtp_status rtp_adamw_destroy(rtp_adamw *opt)
{
    delete opt;
    return RTP_OK;
}

extern "C" rtp_status rtp_adamw_scalars_of(const rtp_adamw_hyper *h, rtp_adamw_scalars *out)
{
    const char *who = "rtp_adamw_scalars_of";
    if (!h || !out) return fail(RTP_ERR_INVALID, "%s: null argument", who);
    if (!(h->beta1 >= 0 && h->beta1 < 1 && h->beta2 >= 0 && h->beta2 < 1) || !((float)h->eps >= FLT_MIN) || !std::isfinite((float)h->eps) ||
        !std::isfinite((float)h->lr) || h->step < 1)
        return fail(RTP_ERR_INVALID, "%s: need 0 <= beta < 1, eps of at least 2^-126, a finite lr, step >= 1", who);
    *out = rtp_adamw_scalars{};
    out->beta1 = (float)h->beta1;
    out->one_minus_beta1 = (float)(1.0 - h->beta1);
    out->beta2 = (float)h->beta2;
    out->one_minus_beta2 = (float)(1.0 - h->beta2);
    out->lr = (float)h->lr;
    out->step_size = (float)(h->lr / (1.0 - std::pow(h->beta1, (double)h->step)));
    out->root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, (double)h->step)));
    out->eps = (float)h->eps;
    out->seed = h->seed;
    return RTP_OK;
}

extern "C" rtp_status rtp_adamw_step(rtp_adamw *opt, const rtp_adamw_hyper *h, const rtp_adamw_scalars *scalars_dev, const float *scale_dev, void *stream)
{
    const char *who = "rtp_adamw_step";
    if (!opt || !h == !scalars_dev) return fail(RTP_ERR_INVALID, "%s: needs an optimizer, and either values or their place in device memory", who);
    if (!aligned(scalars_dev, 16) || !aligned(scale_dev, 4)) return fail(RTP_ERR_SHAPE, "%s: bad alignment", who);
    AdamwArgs a{opt->entries, opt->owner, opt->chunks, opt->m, opt->v, opt->exps, {}, scalars_dev, scale_dev};
    if (h) RTP_TRY(rtp_adamw_scalars_of(h, &a.sc));
    HIP_TRY(launch_adamw(opt->moments, a, (hipStream_t)stream));
    return RTP_OK;
}

extern "C" rtp_status rtp_adamw_moments(const rtp_adamw *opt, rtp_dtype dtype, void *m_out, void *v_out, void *stream)
{
    const char *who = "rtp_adamw_moments";
    if (!opt || !m_out || !v_out) return fail(RTP_ERR_INVALID, "%s: null argument", who);
    if (dtype != RTP_F32 && dtype != RTP_BF16) return fail(RTP_ERR_UNSUPPORTED, "%s: fp32 or bf16", who);
    if (!aligned(m_out, 16) || !aligned(v_out, 16)) return fail(RTP_ERR_SHAPE, "%s: the outputs must be multiples of 16 bytes", who);
    HIP_TRY(launch_adamw_moments(opt->moments, dtype, opt->m, opt->v, opt->exps, opt->blocks, m_out, v_out, (hipStream_t)stream));
    return RTP_OK;
}
