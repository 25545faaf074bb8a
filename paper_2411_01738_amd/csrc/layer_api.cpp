// C ABI of what surrounds the attention in a layer (declared in
// include/xdit.h): rotary tables, rotation, the norms of queries and keys,
// forward and backward, and the attention's gradients.  Checks first, then
// one dispatch.
#include "layer_api.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>

using namespace xdit_api;

namespace {

// One [batch, tokens, heads, head_dim] tensor of a call, by strides in elements.
struct View {
    const void* p;
    int64_t n[3], s[3];  // sizes and strides of batch, token, head
    int64_t d;
    int es;
    const char* name;

    bool empty() const { return n[0] == 0 || n[1] == 0 || n[2] == 0; }
    int64_t bytes() const {  // from the first element to past the last
        if (empty()) return 0;
        return es * ((n[0] - 1) * s[0] + (n[1] - 1) * s[1] + (n[2] - 1) * s[2] + d);
    }
    Span span() const { return {p, bytes(), name}; }
    xdit::HeadView head_view() const { return {p, s[0], s[1], s[2]}; }
};

View view(const void* p, int64_t B, int64_t N, int64_t H, int64_t d, int es, const int64_t* strides, const char* name) {
    View v{p, {B, N, H}, {N * H * d, H * d, d}, d, es, name};
    if (strides)
        for (int i = 0; i < 3; ++i) v.s[i] = strides[i];
    for (int i = 0; i < 3; ++i)
        if (v.n[i] <= 1) v.s[i] = 0;  // never stepped
    return v;
}

int check_view(const View& v) {
    if (v.empty()) return XDIT_OK;
    if (v.p == nullptr) return fail(XDIT_ERR_NULL, "%s is NULL", v.name);
    if (((uintptr_t)v.p & 15u) != 0) return fail(XDIT_ERR_LAYOUT, "%s is not 16-byte aligned", v.name);
    double end = 0;
    for (int i = 0; i < 3; ++i) {
        if (v.s[i] < 0) return fail(XDIT_ERR_LAYOUT, "%s: negative stride", v.name);
        if (v.s[i] * v.es % 16 != 0) return fail(XDIT_ERR_LAYOUT, "%s: strides are multiples of 16 bytes", v.name);
        end += (double)(v.n[i] - 1) * (double)v.s[i];
    }
    if (end > 1099511627776.0) return fail(XDIT_ERR_SHAPE, "%s: tensor too large", v.name);
    return XDIT_OK;
}

// No two elements of an output share memory.
int check_written(const View& v) {
    if (v.empty()) return XDIT_OK;
    int o[3] = {0, 1, 2};
    std::sort(o, o + 3, [&](int a, int b) { return v.s[a] < v.s[b]; });
    int64_t reach = v.d;
    for (int i : o) {
        if (v.n[i] <= 1) continue;
        if (v.s[i] < reach) return fail(XDIT_ERR_ALIAS, "%s overlaps itself", v.name);
        reach = v.s[i] * (v.n[i] - 1) + reach;
    }
    return XDIT_OK;
}

bool same_view(const View& a, const View& b) {
    return a.p == b.p && std::equal(a.n, a.n + 3, b.n) && std::equal(a.s, a.s + 3, b.s);
}

// Length of a view's elements modulo a period, -1 where its longer strides are
// no multiples of it.
int64_t reach_within(const View& v, int64_t period) {
    int64_t r = v.d;
    for (int i = 0; i < 3; ++i) {
        if (v.s[i] < period) r += (v.n[i] - 1) * v.s[i];
        else if (v.s[i] % period != 0) return -1;
    }
    return r;
}

// Whether two views share no element: their spans lie apart, or there is a
// stride of which their elements keep to different parts (heads of one fused
// projection's rows, head-major tensors of one buffer, every other token).
bool apart(const View& a, const View& b) {
    if (!overlap(a.span(), b.span())) return true;
    const int64_t delta = ((intptr_t)b.p - (intptr_t)a.p) / a.es;
    for (const View* v : {&a, &b})
        for (const int64_t period : v->s) {
            if (period <= 0) continue;
            const int64_t ra = reach_within(a, period), rb = reach_within(b, period), r = (delta % period + period) % period;
            if (ra >= 0 && rb >= 0 && r >= ra && r + rb <= period) return true;
        }
    return false;
}

int check_apart(const View& out, const View& in) {
    if (!apart(out, in)) return fail(XDIT_ERR_ALIAS, "%s overlaps %s", out.name, in.name);
    return XDIT_OK;
}

int check_f32(const Span& s) {
    if (s.bytes > 0 && s.p != nullptr && ((uintptr_t)s.p & 3u) != 0)
        return fail(XDIT_ERR_LAYOUT, "%s is not 4-byte aligned", s.name);
    return XDIT_OK;
}

// Checks a rotation's arguments; the tables' spans are for the checks of overlap.
int check_rotation(const char* fn, const float* cos, const float* sin, int64_t rot, int64_t d, int32_t layout,
                   int64_t table_rows, Span* sc, Span* ss) {
    if (layout != XDIT_PAIRS_INTERLEAVED && layout != XDIT_PAIRS_HALF)
        return fail(XDIT_ERR_RANGE, "%s: unknown layout %d", fn, layout);
    if (rot < 0 || rot > d || rot % 8 != 0)
        return fail(XDIT_ERR_SHAPE, "%s: rot_dim = %lld is not a multiple of 8 up to head_dim", fn, (long long)rot);
    *sc = {cos, table_rows * (rot / 2) * 4, "cos"};
    *ss = {sin, table_rows * (rot / 2) * 4, "sin"};
    if (rot == 0 && (cos != nullptr || sin != nullptr))
        return fail(XDIT_ERR_SHAPE, "%s: a table for rot_dim = 0", fn);
    XDIT_TRY(check_ptr(*sc));
    return check_ptr(*ss);
}

int check_heads(const char* fn, int64_t B, int64_t N, int64_t H) {
    XDIT_TRY(check_dims(fn, B, N, 0, H));
    if ((double)B * (double)N >= 2147483648.0) return fail(XDIT_ERR_SHAPE, "%s: more than 2^31 - 1 rows", fn);
    if (H > 65536) return fail(XDIT_ERR_SHAPE, "%s: more than 65536 heads", fn);
    return XDIT_OK;
}

int check_qk(const char* fn, const xdit_qk* p) {
    if (p == nullptr) return fail(XDIT_ERR_NULL, "%s: the parameters are NULL", fn);
    XDIT_TRY(check_dtype_dim(p->dtype, p->head_dim));
    if (p->weight_dtype != XDIT_BF16 && p->weight_dtype != XDIT_F32)
        return fail(XDIT_ERR_DTYPE, "%s: unknown weight_dtype %d", fn, p->weight_dtype);
    XDIT_TRY(check_heads(fn, p->batch, p->tokens, p->q_heads));
    XDIT_TRY(check_heads(fn, p->batch, p->tokens, p->k_heads));
    if (p->norm < XDIT_NORM_NONE || p->norm > XDIT_NORM_LAYER)
        return fail(XDIT_ERR_RANGE, "%s: unknown norm %d", fn, p->norm);
    if (p->norm == XDIT_NORM_NONE && (p->wq || p->wk || p->bq || p->bk || p->rot_dim == 0))
        return fail(XDIT_ERR_RANGE, "%s: without a norm there are no weights, and a rotation", fn);
    if (p->norm == XDIT_NORM_RMS && (p->bq || p->bk)) return fail(XDIT_ERR_RANGE, "%s: the RMS norm has no bias", fn);
    if (!(p->eps >= 0.0) || !std::isfinite((float)p->eps))
        return fail(XDIT_ERR_RANGE, "%s: eps = %g is no float32 number from 0 on", fn, p->eps);
    for (const void* w : {p->wq, p->wk, p->bq, p->bk})
        if (w && ((uintptr_t)w & (p->weight_dtype == XDIT_BF16 ? 1u : 3u)))
            return fail(XDIT_ERR_LAYOUT, "%s: a weight is not aligned to its type", fn);
    Span sc, ss;
    return check_rotation(fn, p->cos, p->sin, p->rot_dim, p->head_dim, p->layout,
                          p->tokens * (p->table_per_batch ? p->batch : 1), &sc, &ss);
}

xdit::NormRopeParams params_of(const xdit_qk& p) {
    xdit::NormRopeParams r{};
    r.side[0].w = p.wq;
    r.side[0].b = p.bq;
    r.side[0].heads = (int)p.q_heads;
    r.side[1].w = p.wk;
    r.side[1].b = p.bk;
    r.side[1].heads = (int)p.k_heads;
    r.cos = p.cos;
    r.sin = p.sin;
    r.table_batch = p.table_per_batch ? p.tokens * (p.rot_dim / 2) : 0;
    r.B = (int)p.batch;
    r.N = (int)p.tokens;
    r.D = (int)p.head_dim;
    r.rot = (int)p.rot_dim;
    r.bf16 = p.dtype == XDIT_BF16;
    r.weight_bf16 = p.weight_dtype == XDIT_BF16;
    r.norm = p.norm;
    r.half = p.layout == XDIT_PAIRS_HALF;
    r.eps = (float)p.eps;
    return r;
}

int64_t align256(int64_t x) { return (x + 255) / 256 * 256; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How the two sweeps of the gradients are cut: their workgroups share one
// launch, and few resident rows over a long other side would leave CUs idle.
struct BwdPlan {
    int q_splits, kv_splits;
    int64_t step;                        // batches of a launch
    int64_t rows_bytes, q_bytes, bytes;  // of the workspace: the rows' scalars, the partials of dq, of dk and dv
};

BwdPlan bwd_plan(int64_t B, int64_t Nq, int64_t Nk, int64_t H, int64_t d, int32_t dtype) {
    BwdPlan p;
    const xdit::BwdSplits s = xdit::bwd_splits(B * H, Nq, Nk, (int)d, dtype == XDIT_BF16);
    p.q_splits = s.q, p.kv_splits = s.kv;
    // a grid holds fewer than 2^32 threads: whole batches at a time, which use
    // the workspace one after another
    const int64_t sweeps = ceil_div(Nq, s.rows) * s.q + ceil_div(Nk, s.rows) * s.kv;
    const int64_t wgs = std::max<int64_t>(1, H * std::max(ceil_div(Nq, 8), sweeps));
    p.step = std::min(B, std::max<int64_t>(1, (((int64_t)1 << 24) - 1) / wgs));
    p.rows_bytes = align256(8 * p.step * H * Nq);
    p.q_bytes = p.q_splits > 1 ? align256(4 * p.q_splits * p.step * Nq * H * d) : 0;
    p.bytes = p.rows_bytes + p.q_bytes + (p.kv_splits > 1 ? align256(8 * p.kv_splits * p.step * Nk * H * d) : 0);
    return p;
}

}  // namespace

namespace xdit_api {

void qk_spans(const xdit_qk& p, Span (&s)[6]) {
    const int64_t n = p.head_dim * (p.weight_dtype == XDIT_BF16 ? 2 : 4);
    const int64_t t = p.tokens * (p.table_per_batch ? p.batch : 1) * (p.rot_dim / 2) * 4;
    s[0] = {p.wq, p.wq ? n : 0, "wq"};
    s[1] = {p.wk, p.wk ? n : 0, "wk"};
    s[2] = {p.bq, p.bq ? n : 0, "bq"};
    s[3] = {p.bk, p.bk ? n : 0, "bk"};
    s[4] = {p.cos, t, "cos"};
    s[5] = {p.sin, t, "sin"};
}

}  // namespace xdit_api

namespace {

// Checks of a forward call; its views in argument order.
int check_forward(const char* fn, const xdit_qk* p, const void* q, const void* k, void* q_out, void* k_out, View (&v)[4]) {
    XDIT_TRY(check_qk(fn, p));
    const int es = esize_of(p->dtype);
    const int64_t *st = p->strides, heads[4] = {p->q_heads, p->k_heads, p->q_heads, p->k_heads};
    const void* ptr[4] = {q, k, q_out, k_out};
    const char* names[4] = {"q", "k", "q_out", "k_out"};
    for (int i = 0; i < 4; ++i) {
        v[i] = view(ptr[i], p->batch, p->tokens, heads[i], p->head_dim, es, st ? st + 3 * i : nullptr, names[i]);
        XDIT_TRY(check_view(v[i]));
    }
    Span sp[6];
    qk_spans(*p, sp);
    for (int o = 2; o < 4; ++o) {
        XDIT_TRY(check_written(v[o]));
        for (int i = 0; i < o; ++i)
            if (i != o - 2 || !same_view(v[o], v[i])) XDIT_TRY(check_apart(v[o], v[i]));
        for (const Span& s : sp) XDIT_TRY(check_no_overlap(v[o].span(), s));
    }
    return XDIT_OK;
}

}  // namespace

namespace xdit_api {

int check_qk_call(const char* fn, const xdit_qk* p, const void* q, const void* k, void* q_out, void* k_out) {
    View v[4];
    return check_forward(fn, p, q, k, q_out, k_out, v);
}

int qk_norm_rope(const char* fn, const xdit_qk* p, const void* q, const void* k, void* q_out, void* k_out) {
    View v[4];
    XDIT_TRY(check_forward(fn, p, q, k, q_out, k_out, v));
    if (p->batch == 0 || p->tokens == 0) return XDIT_OK;
    xdit::NormRopeParams r = params_of(*p);
    for (int i = 0; i < 2; ++i) {
        r.side[i].x = v[i].head_view();
        r.side[i].y = v[2 + i].head_view();
    }
    return hip_status(xdit::launch_norm_rope(r, g_stream), fn);
}

}  // namespace xdit_api

extern "C" {

int xdit_rope_table(const void* pos, int32_t pos_dtype, int64_t n, int32_t n_axes, const int32_t* dims,
                    double theta, const xdit_rope_scaling* scaling, float* cos, float* sin) {
    clear_error();
    const char* fn = "xdit_rope_table";
    if (pos_dtype != XDIT_I64 && pos_dtype != XDIT_F32)
        return fail(XDIT_ERR_DTYPE, "%s: positions are int64 or float32", fn);
    if (n < 0 || n > kMaxDim) return fail(XDIT_ERR_SHAPE, "%s: n = %lld outside [0, 2^31)", fn, (long long)n);
    if (n_axes < 1 || n_axes > XDIT_MAX_AXES)
        return fail(XDIT_ERR_RANGE, "%s: n_axes = %d outside [1, %d]", fn, n_axes, XDIT_MAX_AXES);
    if (dims == nullptr) return fail(XDIT_ERR_NULL, "%s: dims is NULL", fn);
    if (!(theta > 0.0) || !std::isfinite(theta)) return fail(XDIT_ERR_RANGE, "%s: theta = %g is not positive", fn, theta);
    xdit::RopeTableParams p{};
    p.factor = p.magnitude = 1.0;
    p.orig_len = 1.0, p.fast = 32.0, p.slow = 1.0;
    if (scaling) {
        p.scaling = scaling->kind;
        p.magnitude = scaling->magnitude;
        if (p.scaling < XDIT_ROPE_NONE || p.scaling > XDIT_ROPE_RAMP)
            return fail(XDIT_ERR_RANGE, "%s: unknown scaling %d", fn, p.scaling);
        if (!std::isfinite(p.magnitude)) return fail(XDIT_ERR_RANGE, "%s: the magnitude is not finite", fn);
        if (p.scaling != XDIT_ROPE_NONE) p.factor = scaling->factor;
        if (!(p.factor > 0.0) || !std::isfinite(p.factor))
            return fail(XDIT_ERR_RANGE, "%s: factor = %g is not positive", fn, p.factor);
        if (p.scaling == XDIT_ROPE_RAMP) {
            p.orig_len = scaling->orig_len, p.fast = scaling->fast, p.slow = scaling->slow;
            if (!(p.orig_len > 0.0) || !std::isfinite(p.orig_len) || !std::isfinite(p.fast) || !std::isfinite(p.slow) ||
                !(p.fast > p.slow))
                return fail(XDIT_ERR_RANGE, "%s: the ramp needs orig_len > 0 and fast > slow", fn);
        }
    }
    int64_t all = 0;
    for (int a = 0; a < n_axes; ++a) {
        if (dims[a] < 2 || dims[a] % 2 != 0 || dims[a] > 256)
            return fail(XDIT_ERR_SHAPE, "%s: dims[%d] = %d is not an even number from 2 to 256", fn, a, dims[a]);
        if (p.scaling == XDIT_ROPE_NTK && dims[a] == 2)
            return fail(XDIT_ERR_SHAPE, "%s: dims[%d] = 2 has no slowest pair to scale", fn, a);
        p.dims[a] = dims[a];
        all += dims[a];
    }
    if (all > 256) return fail(XDIT_ERR_SHAPE, "%s: %lld dims in all, above 256", fn, (long long)all);
    const Span sp{pos, n * n_axes * (pos_dtype == XDIT_I64 ? 8 : 4), "pos"}, sc{cos, n * all / 2 * 4, "cos"},
        ss{sin, n * all / 2 * 4, "sin"};
    for (const Span* s : {&sp, &sc, &ss}) XDIT_TRY(check_ptr(*s));
    XDIT_TRY(check_no_overlap(sc, sp));
    XDIT_TRY(check_no_overlap(ss, sp));
    XDIT_TRY(check_no_overlap(sc, ss));
    if (n == 0) return XDIT_OK;
    p.pos = pos;
    p.pos_i64 = pos_dtype == XDIT_I64;
    p.axes = n_axes;
    p.theta = theta;
    p.cos = cos;
    p.sin = sin;
    p.n = n;
    return hip_status(xdit::launch_rope_table(p, g_stream), fn);
}

int xdit_rope(const void* x, const float* cos, const float* sin, void* y, const int64_t* strides,
              int64_t batch, int64_t tokens, int64_t heads, int64_t head_dim, int64_t rot_dim,
              int32_t table_per_batch, int32_t layout, int32_t transpose, int32_t dtype) {
    clear_error();
    const char* fn = "xdit_rope";
    XDIT_TRY(check_dtype_dim(dtype, head_dim));
    XDIT_TRY(check_heads(fn, batch, tokens, heads));
    if (rot_dim <= 0) return fail(XDIT_ERR_SHAPE, "%s: rot_dim = %lld", fn, (long long)rot_dim);
    Span sc, ss;
    XDIT_TRY(check_rotation(fn, cos, sin, rot_dim, head_dim, layout, tokens * (table_per_batch ? batch : 1), &sc, &ss));
    const int es = esize_of(dtype);
    const View vx = view(x, batch, tokens, heads, head_dim, es, strides, "x");
    const View vy = view(y, batch, tokens, heads, head_dim, es, strides ? strides + 3 : nullptr, "y");
    XDIT_TRY(check_view(vx));
    XDIT_TRY(check_view(vy));
    XDIT_TRY(check_written(vy));
    if (!same_view(vx, vy)) XDIT_TRY(check_apart(vy, vx));
    XDIT_TRY(check_no_overlap(vy.span(), sc));
    XDIT_TRY(check_no_overlap(vy.span(), ss));
    if (vx.empty()) return XDIT_OK;
    xdit_qk p{};
    p.batch = batch, p.tokens = tokens, p.q_heads = heads, p.head_dim = head_dim;
    p.dtype = dtype, p.weight_dtype = XDIT_F32, p.layout = layout, p.rot_dim = rot_dim;
    p.cos = cos, p.sin = sin, p.table_per_batch = table_per_batch;
    xdit::NormRopeParams r = params_of(p);
    r.side[0].x = vx.head_view();
    r.side[0].y = vy.head_view();
    r.transpose = transpose != 0;
    return hip_status(xdit::launch_norm_rope(r, g_stream), fn);
}

int xdit_qk_norm_rope(const xdit_qk* p, const void* q, const void* k, void* q_out, void* k_out) {
    clear_error();
    return qk_norm_rope("xdit_qk_norm_rope", p, q, k, q_out, k_out);
}

int64_t xdit_qk_norm_rope_bwd_workspace_bytes(int64_t batch, int64_t tokens, int64_t q_heads, int64_t k_heads,
                                              int64_t head_dim, int32_t dtype) {
    clear_error();
    const char* fn = "xdit_qk_norm_rope_bwd_workspace_bytes";
    if (check_dtype_dim(dtype, head_dim) != XDIT_OK || check_heads(fn, batch, tokens, q_heads) != XDIT_OK ||
        check_heads(fn, batch, tokens, k_heads) != XDIT_OK)
        return -1;
    return 4 * xdit::norm_rope_bwd_partials(batch * tokens, (int)q_heads, (int)k_heads, (int)head_dim, dtype == XDIT_BF16);
}

int xdit_qk_norm_rope_bwd(const xdit_qk* p, const void* q, const void* k, const void* dq_out,
                          const void* dk_out, void* dq, void* dk, float* dwq, float* dwk, float* dbq,
                          float* dbk, void* workspace, int64_t workspace_bytes) {
    clear_error();
    const char* fn = "xdit_qk_norm_rope_bwd";
    XDIT_TRY(check_qk(fn, p));
    const int es = esize_of(p->dtype);
    const int64_t* st = p->strides;
    const void* ptr[6] = {q, k, dq_out, dk_out, dq, dk};
    const char* names[6] = {"q", "k", "dq_out", "dk_out", "dq", "dk"};
    View v[6];
    for (int i = 0; i < 6; ++i) {
        v[i] = view(ptr[i], p->batch, p->tokens, i % 2 ? p->k_heads : p->q_heads, p->head_dim, es,
                    st ? st + 3 * i : nullptr, names[i]);
        XDIT_TRY(check_view(v[i]));
    }
    if ((dwq || dwk) && p->norm == XDIT_NORM_NONE) return fail(XDIT_ERR_RANGE, "%s: without a norm there are no weights", fn);
    if ((dbq || dbk) && p->norm != XDIT_NORM_LAYER)
        return fail(XDIT_ERR_RANGE, "%s: only the layer norm has a bias", fn);
    if (p->k_heads == 0 && (dwk || dbk)) return fail(XDIT_ERR_SHAPE, "%s: no keys, but a gradient of their weights", fn);
    Span ins[6];
    qk_spans(*p, ins);
    const bool sums = dwq || dwk || dbq || dbk;
    const int64_t need = sums ? 4 * xdit::norm_rope_bwd_partials(p->batch * p->tokens, (int)p->q_heads, (int)p->k_heads,
                                                                 (int)p->head_dim, p->dtype == XDIT_BF16)
                              : 0;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need))
        return fail(XDIT_ERR_RANGE, "%s: workspace of %lld bytes needed", fn, (long long)need);
    // every output against every input and the other outputs
    const int64_t wb = p->head_dim * 4;
    const Span so[5] = {{dwq, dwq ? wb : 0, "dwq"},
                        {dwk, dwk ? wb : 0, "dwk"},
                        {dbq, dbq ? wb : 0, "dbq"},
                        {dbk, dbk ? wb : 0, "dbk"},
                        {workspace, need, "workspace"}};
    for (int i = 0; i < 4; ++i) XDIT_TRY(check_f32(so[i]));
    XDIT_TRY(check_ptr(so[4]));
    for (int o = 4; o < 6; ++o) {
        XDIT_TRY(check_written(v[o]));
        for (int i = 0; i < o; ++i)
            if (!((i == o - 4 || i == o - 2) && same_view(v[o], v[i]))) XDIT_TRY(check_apart(v[o], v[i]));
        for (const Span& s : ins) XDIT_TRY(check_no_overlap(v[o].span(), s));
    }
    for (int a = 0; a < 5; ++a) {
        for (const View& x : v) XDIT_TRY(check_no_overlap(so[a], x.span()));
        for (const Span& s : ins) XDIT_TRY(check_no_overlap(so[a], s));
        for (int b = 0; b < a; ++b) XDIT_TRY(check_no_overlap(so[a], so[b]));
    }
    xdit::NormRopeParams r = params_of(*p);
    float* grads[2][2] = {{dwq, dbq}, {dwk, dbk}};
    for (int i = 0; i < 2; ++i) {
        r.side[i].x = v[i].head_view();
        r.side[i].g = v[2 + i].head_view();
        r.side[i].y = v[4 + i].head_view();
        r.side[i].dw = grads[i][0];
        r.side[i].db = grads[i][1];
    }
    r.part = (float*)workspace;
    if (p->norm != XDIT_NORM_NONE) return hip_status(xdit::launch_norm_rope_bwd(r, g_stream), fn);
    // the rotation alone: the gradients turned back
    if (p->batch == 0 || p->tokens == 0) return XDIT_OK;
    r.side[0].x = r.side[0].g;
    r.side[1].x = r.side[1].g;
    r.transpose = 1;
    return hip_status(xdit::launch_norm_rope(r, g_stream), fn);
}

int64_t xdit_chunk_attn_bwd_workspace_bytes(int64_t batch, int64_t q_len, int64_t kv_len, int64_t heads,
                                            int64_t head_dim, int32_t dtype) {
    clear_error();
    const char* fn = "xdit_chunk_attn_bwd_workspace_bytes";
    if (check_dtype_dim(dtype, head_dim) != XDIT_OK || check_dims(fn, batch, q_len, kv_len, heads) != XDIT_OK) return -1;
    return bwd_plan(batch, q_len, kv_len, heads, head_dim, dtype).bytes;
}

int xdit_chunk_attn_bwd(const void* q, const void* k, const void* v, const void* out, const float* lse,
                        const void* dout, const float* dlse, void* dq, void* dk, void* dv, int32_t accum,
                        void* workspace, int64_t workspace_bytes, int64_t batch, int64_t q_len,
                        int64_t kv_len, int64_t heads, int64_t head_dim, int32_t dtype) {
    clear_error();
    const char* fn = "xdit_chunk_attn_bwd";
    XDIT_TRY(check_dtype_dim(dtype, head_dim));
    XDIT_TRY(check_dims(fn, batch, q_len, kv_len, heads));
    const int es = esize_of(dtype);
    XDIT_TRY(check_batch_bytes(fn, std::max(q_len, kv_len), heads, head_dim, es));
    if (accum & ~(XDIT_ACCUM_DQ | XDIT_ACCUM_DKV)) return fail(XDIT_ERR_RANGE, "%s: unknown accum %d", fn, accum);
    const int eq = accum & XDIT_ACCUM_DQ ? 4 : es, ek = accum & XDIT_ACCUM_DKV ? 4 : es;
    const int64_t nq = batch * q_len * heads, nk = batch * kv_len * heads;
    const Span sq{q, nq * head_dim * es, "q"}, sk{k, nk * head_dim * es, "k"}, sv{v, nk * head_dim * es, "v"},
        so{out, nq * head_dim * es, "out"}, sl{lse, nq * 4, "lse"}, sg{dout, nq * head_dim * es, "dout"},
        se{dlse, dlse ? nq * 4 : 0, "dlse"};
    const Span gq{dq, nq * head_dim * eq, "dq"}, gk{dk, nk * head_dim * ek, "dk"}, gv{dv, nk * head_dim * ek, "dv"};
    for (const Span* s : {&sq, &sk, &sv, &so, &sg, &gq, &gk, &gv}) XDIT_TRY(check_ptr(*s));
    if (nq > 0 && lse == nullptr) return fail(XDIT_ERR_NULL, "lse is NULL");
    XDIT_TRY(check_f32(sl));
    XDIT_TRY(check_f32(se));
    const BwdPlan plan = bwd_plan(batch, q_len, kv_len, heads, head_dim, dtype);
    if (plan.bytes > 0 && (workspace == nullptr || workspace_bytes < plan.bytes))
        return fail(XDIT_ERR_RANGE, "%s: workspace of %lld bytes needed", fn, (long long)plan.bytes);
    if (plan.bytes > 0 && ((uintptr_t)workspace & 255u)) return fail(XDIT_ERR_LAYOUT, "%s: workspace is not 256-byte aligned", fn);
    const Span sw{workspace, plan.bytes, "workspace"};
    const Span* outs[] = {&gq, &gk, &gv, &sw};
    for (int i = 0; i < 4; ++i) {
        for (const Span* s : {&sq, &sk, &sv, &so, &sl, &sg, &se}) XDIT_TRY(check_no_overlap(*outs[i], *s));
        for (int j = 0; j < i; ++j) XDIT_TRY(check_no_overlap(*outs[i], *outs[j]));
    }
    if (batch == 0 || heads == 0) return XDIT_OK;
    for (int64_t b0 = 0; b0 < batch; b0 += plan.step) {
        auto at = [&](const void* p, int64_t rows, int bytes) -> char* {
            return p ? (char*)const_cast<void*>(p) + b0 * rows * heads * bytes : nullptr;
        };
        xdit::AttnBwdParams p{};
        const int d = (int)head_dim;
        p.q = at(q, q_len, es * d), p.k = at(k, kv_len, es * d), p.v = at(v, kv_len, es * d);
        p.out = at(out, q_len, es * d), p.dout = at(dout, q_len, es * d);
        p.lse = (const float*)at(lse, q_len, 4), p.dlse = (const float*)at(dlse, q_len, 4);
        p.dq = at(dq, q_len, eq * d), p.dk = at(dk, kv_len, ek * d), p.dv = at(dv, kv_len, ek * d);
        p.B = (int)std::min(plan.step, batch - b0), p.H = (int)heads, p.Nq = (int)q_len, p.Nk = (int)kv_len, p.D = d;
        p.bf16 = dtype == XDIT_BF16;
        p.accum_q = (accum & XDIT_ACCUM_DQ) != 0, p.accum_kv = (accum & XDIT_ACCUM_DKV) != 0;
        p.q_splits = plan.q_splits, p.kv_splits = plan.kv_splits;
        p.rows = (float*)workspace;
        p.q_part = (float*)((char*)workspace + plan.rows_bytes);
        p.kv_part = (float*)((char*)workspace + plan.rows_bytes + plan.q_bytes);
        XDIT_TRY(hip_status(xdit::launch_bwd_rows(p, g_stream), fn));
        XDIT_TRY(hip_status((p.bf16 ? xdit::launch_attn_bwd_bf16 : xdit::launch_attn_bwd_f32)(p, g_stream), fn));
        XDIT_TRY(hip_status(xdit::launch_bwd_join(p, g_stream), fn));
    }
    return XDIT_OK;
}

}  // extern "C"
