// The torch binding's call path in native code: checks the tensors of a call,
// reads their sizes and pointers, sets torch's current stream and calls the
// library (include/xdit.h).  A function returns the library's status, or None
// when an argument is not what its fast path takes (another type, shape,
// layout or device): the caller then goes through the checks in Python, which
// name what is wrong.  A call through Python attribute reads and ctypes took
// 8 to 12 us of host time, more than the shortest kernels run; this path
// takes about 2 us plus the launch.
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/xdit.h"

namespace {

PyObject* g_device = nullptr;      // () -> index of the current device
PyObject* g_raw_stream = nullptr;  // (index) -> raw handle of torch's current stream

// One tensor argument: dense, strided, on the GPU.
struct T {
    void* p = nullptr;
    at::IntArrayRef s;
    at::ScalarType dt = at::kFloat;
    int64_t bytes = 0;
};

bool get(PyObject* o, int64_t dims, T* t) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& x = THPVariable_Unpack(o);
    if (x.layout() != at::kStrided || !x.is_cuda() || (dims >= 0 && x.dim() != dims) || !x.is_contiguous()) return false;
    t->s = x.sizes();
    t->dt = x.scalar_type();
    t->p = x.data_ptr();
    t->bytes = x.numel() * (int64_t)x.element_size();
    return true;
}

// a K/V buffer: K's plane, then V's
bool buffer(PyObject* o, T* t) { return get(o, 5, t) && t->s[0] >= 2; }

bool get_or_none(PyObject* o, int64_t dims, T* t) { return o == Py_None || get(o, dims, t); }

bool shape4(const T& t, at::ScalarType dt, int64_t a, int64_t b, int64_t c, int64_t d) {
    return t.dt == dt && t.s[0] == a && t.s[1] == b && t.s[2] == c && t.s[3] == d;
}

// an LSE of B x H x n, or none given
bool is_lse(const T& t, int64_t B, int64_t H, int64_t n) {
    return t.s.empty() || (t.dt == at::kFloat && t.s[0] == B && t.s[1] == H && t.s[2] == n);
}

bool code(at::ScalarType dt, int32_t* c) {
    *c = dt == at::kBFloat16 ? XDIT_BF16 : XDIT_F32;
    return dt == at::kBFloat16 || dt == at::kFloat;
}

bool integer(PyObject* o, int64_t* x) {
    if (!PyLong_CheckExact(o)) return false;
    *x = PyLong_AsLongLong(o);
    if (*x == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// a float or a whole number that a double holds
bool number(PyObject* o, double* x) {
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
    *x = PyFloat_AsDouble(o);
    if (*x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// up to XDIT_MAX_RANGES (offset, length) pairs; *F their total length
bool ranges(PyObject* o, int64_t* off, int64_t* len, int32_t* n, int64_t* F) {
    if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) return false;
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(o);
    if (k > XDIT_MAX_RANGES) return false;
    *F = 0;
    for (Py_ssize_t i = 0; i < k; ++i) {
        PyObject* r = PySequence_Fast_GET_ITEM(o, i);
        if (!PyTuple_CheckExact(r) || PyTuple_GET_SIZE(r) != 2) return false;
        if (!integer(PyTuple_GET_ITEM(r, 0), off + i) || !integer(PyTuple_GET_ITEM(r, 1), len + i)) return false;
        *F += len[i];
    }
    *n = (int32_t)k;
    return true;
}

// torch's current stream for the calling thread's launches
bool use_current_stream() {
    PyObject* dev = PyObject_CallNoArgs(g_device);
    PyObject* st = dev ? PyObject_CallOneArg(g_raw_stream, dev) : nullptr;
    Py_XDECREF(dev);
    void* h = st ? PyLong_AsVoidPtr(st) : nullptr;
    Py_XDECREF(st);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    xdit_set_stream(h);
    return true;
}

// Runs `call` without the interpreter lock, as ctypes does.
template <typename F>
PyObject* run(F&& call) {
    if (!use_current_stream()) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// A C++ exception (a tensor without storage, symbolic sizes) leaves the call
// to the Python path.
template <PyObject* (*F)(PyObject* const*)>
PyObject* guarded(PyObject* const* a) {
    try {
        return F(a);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", N, n);
        return nullptr;
    }
    return guarded<F>(a);
}

struct Chunk {
    T q, k, v, out, lse;
    int64_t B, Nq, H, d, Nk;
    int32_t dt;
};

bool chunk_args(PyObject* const* a, bool need_lse, Chunk* c) {
    if (!get(a[0], 4, &c->q) || !get(a[1], 4, &c->k) || !get(a[2], 4, &c->v) || !get(a[3], 4, &c->out) ||
        !get_or_none(a[4], 3, &c->lse) || (need_lse && a[4] == Py_None) || !code(c->q.dt, &c->dt))
        return false;
    c->B = c->q.s[0], c->Nq = c->q.s[1], c->H = c->q.s[2], c->d = c->q.s[3], c->Nk = c->k.s[1];
    return shape4(c->k, c->q.dt, c->B, c->Nk, c->H, c->d) && shape4(c->v, c->q.dt, c->B, c->Nk, c->H, c->d) &&
           shape4(c->out, c->q.dt, c->B, c->Nq, c->H, c->d) && is_lse(c->lse, c->B, c->H, c->Nq);
}

// q, k, v, out, lse, accum
PyObject* chunk(PyObject* const* a) {
    Chunk c;
    const bool accum = a[5] == Py_True;
    if (!chunk_args(a, accum, &c)) Py_RETURN_NONE;
    return run([&] {
        return accum ? xdit_chunk_attn_accum(c.q.p, c.k.p, c.v.p, c.out.p, (float*)c.lse.p, c.B, c.Nq, c.Nk, c.H, c.d, c.dt)
                     : xdit_chunk_attn(c.q.p, c.k.p, c.v.p, c.out.p, (float*)c.lse.p, c.B, c.Nq, c.Nk, c.H, c.d, c.dt);
    });
}

// q, k, v, out, lse, splits, workspace, accum
PyObject* chunk_split(PyObject* const* a) {
    Chunk c;
    T ws;
    int64_t splits;
    const bool accum = a[7] == Py_True;
    if (!chunk_args(a, accum, &c) || !integer(a[5], &splits) || splits != (int32_t)splits || !get_or_none(a[6], -1, &ws))
        Py_RETURN_NONE;
    return run([&] {
        return (accum ? xdit_chunk_attn_accum_split : xdit_chunk_attn_split)(
            c.q.p, c.k.p, c.v.p, c.out.p, (float*)c.lse.p, (int32_t)splits, ws.p, ws.bytes, c.B, c.Nq, c.Nk, c.H, c.d, c.dt);
    });
}

// q, kv_buf, patch_off, patch_len, fresh_k, fresh_v, out
PyObject* patch(PyObject* const* a) {
    T q, kv, fk, fv, out;
    int64_t off, len;
    int32_t dt;
    if (!get(a[0], 4, &q) || !buffer(a[1], &kv) || !integer(a[2], &off) || !integer(a[3], &len) || !get(a[4], 4, &fk) ||
        !get(a[5], 4, &fv) || !get(a[6], 4, &out) || !code(kv.dt, &dt))
        Py_RETURN_NONE;
    const int64_t B = kv.s[1], N = kv.s[2], H = kv.s[3], d = kv.s[4];
    for (const T* t : {&q, &fk, &fv, &out})
        if (!shape4(*t, kv.dt, B, len, H, d)) Py_RETURN_NONE;
    return run([&] { return xdit_patch_attn(q.p, kv.p, off, len, fk.p, fv.p, out.p, B, N, H, d, dt); });
}

// q, kv_buf, ranges, fresh_k, fresh_v, out, lse; SPLIT: then splits, workspace
template <bool SPLIT>
PyObject* general_patch(PyObject* const* a) {
    T q, kv, fk, fv, out, lse, ws;
    int64_t off[XDIT_MAX_RANGES] = {}, len[XDIT_MAX_RANGES] = {}, F, splits = 0;
    int32_t dt, nr;
    if (!get(a[0], 4, &q) || !buffer(a[1], &kv) || !ranges(a[2], off, len, &nr, &F) || !get(a[3], 4, &fk) ||
        !get(a[4], 4, &fv) || !get(a[5], 4, &out) || !get_or_none(a[6], 3, &lse) || !code(kv.dt, &dt) ||
        (SPLIT && (!integer(a[7], &splits) || splits != (int32_t)splits || !get_or_none(a[8], -1, &ws))))
        Py_RETURN_NONE;
    const int64_t Nq = q.s[1], B = kv.s[1], N = kv.s[2], H = kv.s[3], d = kv.s[4];
    if (!shape4(q, kv.dt, B, Nq, H, d) || !shape4(out, kv.dt, B, Nq, H, d) || !shape4(fk, kv.dt, B, F, H, d) ||
        !shape4(fv, kv.dt, B, F, H, d) || !is_lse(lse, B, H, Nq))
        Py_RETURN_NONE;
    return run([&] {
        return SPLIT ? xdit_patch_attn_split(q.p, Nq, kv.p, nr, off, len, fk.p, fv.p, out.p, (float*)lse.p,
                                             (int32_t)splits, ws.p, ws.bytes, B, N, H, d, dt)
                     : xdit_patch_attn_ranges(q.p, Nq, kv.p, nr, off, len, fk.p, fv.p, out.p, (float*)lse.p, B, N, H, d,
                                              dt);
    });
}

constexpr auto patch_ranges = general_patch<false>;
constexpr auto patch_split = general_patch<true>;

// outs, lses, n, out, lse_out
PyObject* merge(PyObject* const* a) {
    T out, lo;
    int64_t n;
    int32_t dt;
    if (!PyList_CheckExact(a[0]) || !PyList_CheckExact(a[1]) || !integer(a[2], &n) || n < 1 || n > XDIT_MAX_PARTIALS ||
        n > PyList_GET_SIZE(a[0]) || n > PyList_GET_SIZE(a[1]) || !get(a[3], 4, &out) || !get_or_none(a[4], 3, &lo) ||
        !code(out.dt, &dt))
        Py_RETURN_NONE;
    const int64_t B = out.s[0], Nq = out.s[1], H = out.s[2], d = out.s[3];
    const void* o[XDIT_MAX_PARTIALS];
    const float* l[XDIT_MAX_PARTIALS];
    for (int64_t r = 0; r < n; ++r) {
        T x, y;
        if (!get(PyList_GET_ITEM(a[0], r), 4, &x) || !get(PyList_GET_ITEM(a[1], r), 3, &y) ||
            !shape4(x, out.dt, B, Nq, H, d) || !is_lse(y, B, H, Nq))
            Py_RETURN_NONE;
        o[r] = x.p;
        l[r] = (const float*)y.p;
    }
    if (!is_lse(lo, B, H, Nq)) Py_RETURN_NONE;
    return run([&] { return xdit_lse_merge(o, l, (int32_t)n, out.p, (float*)lo.p, B, Nq, H, d, dt); });
}

// kv_buf, patch_off, patch_len, fresh_k, fresh_v
PyObject* update(PyObject* const* a) {
    T kv, fk, fv;
    int64_t off, len;
    int32_t dt;
    if (!buffer(a[0], &kv) || !integer(a[1], &off) || !integer(a[2], &len) || !get(a[3], 4, &fk) ||
        !get(a[4], 4, &fv) || !code(kv.dt, &dt))
        Py_RETURN_NONE;
    const int64_t B = kv.s[1], N = kv.s[2], H = kv.s[3], d = kv.s[4];
    if (!shape4(fk, kv.dt, B, len, H, d) || !shape4(fv, kv.dt, B, len, H, d)) Py_RETURN_NONE;
    return run([&] { return xdit_kv_update(kv.p, off, len, fk.p, fv.p, B, N, H, d, dt); });
}

// One [B, N, H, d] tensor argument of any strides whose heads lie contiguous.
struct V : T {
    at::IntArrayRef st;
    c10::DeviceIndex dev = -1;
};

bool view(PyObject* o, V* t) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& x = THPVariable_Unpack(o);
    if (x.layout() != at::kStrided || !x.is_cuda() || x.dim() != 4 || x.stride(3) != 1) return false;
    t->s = x.sizes();
    t->st = x.strides();
    t->dt = x.scalar_type();
    t->p = x.data_ptr();
    t->dev = x.device().index();
    return true;
}

bool like(const V& t, const V& q, int64_t H) {
    return t.dev == q.dev && shape4(t, q.dt, q.s[0], q.s[1], H, q.s[3]);
}

// one of the names, as its place in the list
template <size_t N>
bool choice(PyObject* o, const char* const (&names)[N], int32_t first, int32_t* c) {
    if (!PyUnicode_CheckExact(o)) return false;
    for (size_t i = 0; i < N; ++i)
        if (PyUnicode_CompareWithASCIIString(o, names[i]) == 0) {
            *c = first + (int32_t)i;
            return true;
        }
    return false;
}
const char* const kNorms[] = {"none", "rms", "layer"};
const char* const kLayouts[] = {"interleaved", "half"};

bool device_of(PyObject* o, c10::DeviceIndex dev) { return THPVariable_Unpack(o).device().index() == dev; }

// a dense tensor of the given device, or None
bool on_device(PyObject* o, int64_t dims, c10::DeviceIndex dev, T* t) {
    return o == Py_None || (get(o, dims, t) && device_of(o, dev));
}

// a rotary table of [N, r] or [B, N, r], or none
bool table(PyObject* co, PyObject* so, const V& x, T* c, T* s, int64_t* rot, int32_t* per_batch) {
    if (co == Py_None && so == Py_None) {
        *rot = 0;
        *per_batch = 0;
        return true;
    }
    if (!get(co, -1, c) || !get(so, -1, s) || !device_of(co, x.dev) || !device_of(so, x.dev) || c->dt != at::kFloat ||
        s->dt != at::kFloat || c->s != s->s)
        return false;
    const size_t n = c->s.size();
    if (n != 2 && n != 3) return false;
    if (c->s[n - 2] != x.s[1] || (n == 3 && c->s[0] != x.s[0])) return false;
    *rot = 2 * c->s[n - 1];
    *per_batch = n == 3;
    return true;
}

// the device whose stream the call goes to
bool current_device(c10::DeviceIndex* dev) {
    PyObject* o = PyObject_CallNoArgs(g_device);
    const long d = o ? PyLong_AsLong(o) : -1;
    Py_XDECREF(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    *dev = (c10::DeviceIndex)d;
    return true;
}

const char* const kScalings[] = {"none", "linear", "ntk", "ramp"};

// pos, dims, cos, sin, theta, scaling, factor, orig_len, fast, slow, magnitude
PyObject* rope_table(PyObject* const* a) {
    T pos, c, s;
    c10::DeviceIndex dev;
    xdit_rope_scaling sc{};
    double f[6];
    if (!get(a[0], 2, &pos) || !get(a[2], 2, &c) || !get(a[3], 2, &s) || !PyList_CheckExact(a[1]) || !current_device(&dev) ||
        !device_of(a[0], dev) || !device_of(a[2], dev) || !device_of(a[3], dev) || !choice(a[5], kScalings, 0, &sc.kind))
        Py_RETURN_NONE;
    const int at[6] = {4, 6, 7, 8, 9, 10};
    for (int i = 0; i < 6; ++i)
        if (!number(a[at[i]], &f[i])) Py_RETURN_NONE;
    sc.factor = f[1], sc.orig_len = f[2], sc.fast = f[3], sc.slow = f[4], sc.magnitude = f[5];
    const Py_ssize_t axes = PyList_GET_SIZE(a[1]);
    int32_t dims[XDIT_MAX_AXES];
    int64_t all = 0;
    if (axes < 1 || axes > XDIT_MAX_AXES) Py_RETURN_NONE;
    for (Py_ssize_t i = 0; i < axes; ++i) {
        int64_t d;
        if (!integer(PyList_GET_ITEM(a[1], i), &d) || d < 0 || d > 256) Py_RETURN_NONE;
        dims[i] = (int32_t)d;
        all += d;
    }
    const int64_t n = pos.s[0];
    if (pos.s[1] != axes || (pos.dt != at::kLong && pos.dt != at::kFloat)) Py_RETURN_NONE;
    for (const T* t : {&c, &s})
        if (t->dt != at::kFloat || t->s[0] != n || t->s[1] != all / 2) Py_RETURN_NONE;
    return run([&] {
        return xdit_rope_table(pos.p, pos.dt == at::kLong ? XDIT_I64 : XDIT_F32, n, (int32_t)axes, dims, f[0], &sc, (float*)c.p,
                               (float*)s.p);
    });
}

// x, cos, sin, y, layout, transpose
PyObject* rope(PyObject* const* a) {
    V x, y;
    T c, s;
    int64_t rot;
    int32_t dt, lay, pb;
    c10::DeviceIndex dev;
    if (!view(a[0], &x) || !view(a[3], &y) || !like(y, x, x.s[2]) || !code(x.dt, &dt) || a[1] == Py_None ||
        !table(a[1], a[2], x, &c, &s, &rot, &pb) || !choice(a[4], kLayouts, 0, &lay) || !PyBool_Check(a[5]) ||
        !current_device(&dev) || dev != x.dev)
        Py_RETURN_NONE;
    const int64_t st[6] = {x.st[0], x.st[1], x.st[2], y.st[0], y.st[1], y.st[2]};
    const int32_t tr = a[5] == Py_True;
    return run([&] {
        return xdit_rope(x.p, (const float*)c.p, (const float*)s.p, y.p, st, x.s[0], x.s[1], x.s[2], x.s[3], rot, pb, lay, tr,
                         dt);
    });
}

// The parameters of a call on queries and keys: norm, eps, wq, wk, bq, bk, cos,
// sin, layout at the given places; bq, bk: nullptr where the call has none.
bool qk_params(const V& q, const V& k, PyObject* norm, PyObject* eps, PyObject* const (&w)[4], PyObject* co, PyObject* so,
               PyObject* layout, xdit_qk* p) {
    T c, s, wt[4];
    c10::DeviceIndex dev;
    if (!code(q.dt, &p->dtype) || !choice(norm, kNorms, XDIT_NORM_NONE, &p->norm) || !choice(layout, kLayouts, 0, &p->layout) ||
        !number(eps, &p->eps) || !table(co, so, q, &c, &s, &p->rot_dim, &p->table_per_batch) || !current_device(&dev) ||
        dev != q.dev)
        return false;
    p->weight_dtype = -1;
    for (int i = 0; i < 4; ++i) {
        if (w[i] == nullptr || w[i] == Py_None) continue;
        int32_t wc;
        if (!get(w[i], 1, &wt[i]) || !device_of(w[i], q.dev) || wt[i].s[0] != q.s[3] || !code(wt[i].dt, &wc) ||
            (p->weight_dtype >= 0 && p->weight_dtype != wc))
            return false;
        p->weight_dtype = wc;
    }
    if (p->weight_dtype < 0) p->weight_dtype = XDIT_F32;
    p->batch = q.s[0], p->tokens = q.s[1], p->q_heads = q.s[2], p->head_dim = q.s[3];
    p->k_heads = k.p == nullptr && k.s.empty() ? 0 : k.s[2];
    p->wq = wt[0].p, p->wk = wt[1].p, p->bq = wt[2].p, p->bk = wt[3].p;
    p->cos = (const float*)c.p, p->sin = (const float*)s.p;
    return true;
}

// queries' and keys' tensors in argument order; keys' are all None or all given
template <int N>
bool qk_views(PyObject* const* a, V (&v)[N], int64_t (&st)[3 * N]) {
    const bool keys = a[1] != Py_None;
    for (int i = 0; i < N; ++i) {
        for (int j = 0; j < 3; ++j) st[3 * i + j] = 0;
        if (i % 2 == 1 && !keys) {
            if (a[i] != Py_None) return false;
            continue;
        }
        if (!view(a[i], &v[i]) || !like(v[i], v[0], v[i % 2].s[2])) return false;
        for (int j = 0; j < 3; ++j) st[3 * i + j] = v[i].st[j];
    }
    return true;
}

// q, k, q_out, k_out, norm, eps, wq, wk, bq, bk, cos, sin, layout
PyObject* qk_norm_rope(PyObject* const* a) {
    V v[4];
    int64_t st[12];
    xdit_qk p{};
    PyObject* const w[4] = {a[6], a[7], a[8], a[9]};
    if (!qk_views(a, v, st) || !qk_params(v[0], v[1], a[4], a[5], w, a[10], a[11], a[12], &p)) Py_RETURN_NONE;
    p.strides = st;
    return run([&] { return xdit_qk_norm_rope(&p, v[0].p, v[1].p, v[2].p, v[3].p); });
}

// q, k, dq_out, dk_out, dq, dk, norm, eps, wq, wk, cos, sin, layout, dwq, dwk, dbq, dbk, workspace
PyObject* qk_norm_rope_bwd(PyObject* const* a) {
    V v[6];
    T g[4], ws;
    int64_t st[18];
    xdit_qk p{};
    PyObject* const w[4] = {a[8], a[9], nullptr, nullptr};
    if (!qk_views(a, v, st) || !qk_params(v[0], v[1], a[6], a[7], w, a[10], a[11], a[12], &p)) Py_RETURN_NONE;
    for (int i = 0; i < 4; ++i)
        if (!on_device(a[13 + i], 1, v[0].dev, &g[i]) ||
            (a[13 + i] != Py_None && (g[i].dt != at::kFloat || g[i].s[0] != p.head_dim)))
            Py_RETURN_NONE;
    if (!on_device(a[17], -1, v[0].dev, &ws)) Py_RETURN_NONE;
    p.strides = st;
    return run([&] {
        return xdit_qk_norm_rope_bwd(&p, v[0].p, v[1].p, v[2].p, v[3].p, v[4].p, v[5].p, (float*)g[0].p, (float*)g[1].p,
                                     (float*)g[2].p, (float*)g[3].p, ws.p, ws.bytes);
    });
}

// q, k, v, out, lse, dout, dq, dk, dv, dlse, accum_dq, accum_dkv, workspace
PyObject* chunk_bwd(PyObject* const* a) {
    Chunk c;
    T dout, dq, dk, dv, dlse, ws;
    c10::DeviceIndex dev;
    if (!chunk_args(a, true, &c) || !current_device(&dev) || !get(a[5], 4, &dout) || !get(a[6], 4, &dq) ||
        !get(a[7], 4, &dk) || !get(a[8], 4, &dv) || !get_or_none(a[9], 3, &dlse) || !PyBool_Check(a[10]) ||
        !PyBool_Check(a[11]) || !get_or_none(a[12], -1, &ws))
        Py_RETURN_NONE;
    for (int i : {0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 12})
        if (a[i] != Py_None && !device_of(a[i], dev)) Py_RETURN_NONE;
    const bool aq = a[10] == Py_True, ak = a[11] == Py_True;
    const at::ScalarType t = c.q.dt, tq = aq ? at::kFloat : t, tk = ak ? at::kFloat : t;
    if (!shape4(dout, t, c.B, c.Nq, c.H, c.d) || !shape4(dq, tq, c.B, c.Nq, c.H, c.d) ||
        !shape4(dk, tk, c.B, c.Nk, c.H, c.d) || !shape4(dv, tk, c.B, c.Nk, c.H, c.d) || !is_lse(dlse, c.B, c.H, c.Nq))
        Py_RETURN_NONE;
    return run([&] {
        return xdit_chunk_attn_bwd(c.q.p, c.k.p, c.v.p, c.out.p, (const float*)c.lse.p, dout.p, (const float*)dlse.p, dq.p,
                                   dk.p, dv.p, (aq ? XDIT_ACCUM_DQ : 0) | (ak ? XDIT_ACCUM_DKV : 0), ws.p, ws.bytes, c.B,
                                   c.Nq, c.Nk, c.H, c.d, c.dt);
    });
}

// device, raw_stream: the callables that give torch's current stream
PyObject* init(PyObject* const* a) {
    Py_INCREF(a[0]);
    Py_INCREF(a[1]);
    Py_XSETREF(g_device, a[0]);
    Py_XSETREF(g_raw_stream, a[1]);
    Py_RETURN_NONE;
}

#define ENTRY(name, n) {#name, (PyCFunction)(void (*)(void))&entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(init, 2),         ENTRY(chunk, 6),       ENTRY(chunk_split, 8),
                         ENTRY(patch, 7),        ENTRY(patch_ranges, 7), ENTRY(patch_split, 9),
                         ENTRY(merge, 5),        ENTRY(update, 5),      ENTRY(rope_table, 11), ENTRY(rope, 6),
                         ENTRY(qk_norm_rope, 13), ENTRY(qk_norm_rope_bwd, 18), ENTRY(chunk_bwd, 13),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
