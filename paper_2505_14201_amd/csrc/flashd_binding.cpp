// The marshalling of flashd.py's entry points of the serving path in C++: from the tensors
// to the C call, a call costs 0.4 us of host time here and 3.5 in Python, of which a call on a
// small problem takes 2.5 us more for the launch and the GPU not much longer.
//
// Each function returns the status of the C call, or None where it finds anything out of the ordinary
// (an argument that is no plain GPU tensor of the right type and shape, another current device, a
// stream handed in): nothing has been enqueued then, and the Python form of the same function takes the
// call, with all its checks and messages.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "../../include/flashd.h"

namespace {

using attn_fwd_t = int (*)(const void*, const void*, const void*, void*, int, int, int, int, int, int, int, float,
                           int, void*);
using attn_fwd_kv8_t = int (*)(const void*, const void*, const void*, void*, int, int, int, int, int, int, int,
                               float, float, float, int, void*);
using attn_fwd_state_t = int (*)(const void*, const void*, const void*, void*, const float*, float*, int, int, int,
                                 int, int, int, int, int, float, int, void*);

attn_fwd_t g_attn_fwd = nullptr;
attn_fwd_kv8_t g_attn_fwd_kv8 = nullptr;
attn_fwd_state_t g_attn_fwd_state = nullptr;
PyObject* g_current_device = nullptr;       // () -> index
PyObject* g_raw_stream = nullptr;           // (index) -> handle

// A plain contiguous GPU tensor of four dimensions, or nullptr
const at::Tensor* plain(PyObject* x) {
    if (!THPVariable_CheckExact(x)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(x);
    return t.is_cuda() && t.layout() == at::kStrided && t.dim() == 4 && t.is_contiguous() ? &t : nullptr;
}

// the library's number of a storage type, or -1
int dtype_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
    case at::kFloat: return 0;
    case at::kHalf: return 1;
    case at::kBFloat16: return 2;
    default: return -1;
    }
}

struct Shape { int B, Hq, Hkv, Lq, Lk, d; };

// (sizes that do not fit the C call's ints go to the Python form, which passes them as it always has)
bool shape_of(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, Shape& s) {
    const auto qs = q.sizes(), ks = k.sizes();
    if (qs[0] != ks[0] || qs[3] != ks[3] || v.sizes() != ks) return false;
    for (const int64_t n : {qs[0], qs[1], qs[2], qs[3], ks[1], ks[2]})
        if (n > 0x7fffffff) return false;
    s = {(int)qs[0], (int)qs[1], (int)ks[1], (int)qs[2], (int)ks[2], (int)qs[3]};
    return true;
}

// The handle of the current stream of q's device, which must be the current one.
bool current_stream(const at::Tensor& q, void** stream) {
    PyObject* now = PyObject_CallNoArgs(g_current_device);
    if (now == nullptr) return false;
    const bool here = PyLong_AsLong(now) == q.get_device();
    PyObject* raw = here ? PyObject_CallOneArg(g_raw_stream, now) : nullptr;
    Py_DECREF(now);
    if (raw == nullptr) return false;
    *stream = PyLong_AsVoidPtr(raw);
    Py_DECREF(raw);
    return PyErr_Occurred() == nullptr;
}

bool number(PyObject* x, float* out) {
    const double v = PyFloat_AsDouble(x);
    *out = (float)v;
    return !(v == -1.0 && PyErr_Occurred());
}

PyObject* other_form() {
    PyErr_Clear();
    Py_RETURN_NONE;
}

// (q, k, v, o, causal, scale)
PyObject* py_attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (n != 6) return other_form();
        const at::Tensor *q = plain(a[0]), *k = plain(a[1]), *v = plain(a[2]), *o = plain(a[3]);
        Shape s;
        float scale;
        void* stream;
        if (!q || !k || !v || !o || !shape_of(*q, *k, *v, s) || o->sizes() != q->sizes()) return other_form();
        const int dt = dtype_of(*q);
        if (dt < 0 || k->scalar_type() != q->scalar_type() || v->scalar_type() != q->scalar_type() ||
            o->scalar_type() != q->scalar_type())
            return other_form();
        const int causal = PyObject_IsTrue(a[4]);
        if (causal < 0 || !number(a[5], &scale) || !current_stream(*q, &stream)) return other_form();
        void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr(), *op = o->data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_attn_fwd(qp, kp, vp, op, s.B, s.Hq, s.Hkv, s.Lq, s.Lk, s.d, causal, scale, dt, stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (...) {
        return other_form();
    }
}

// (q, k8, v8, o, causal, scale, kscale, vscale)
PyObject* py_attn_fwd_kv8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (n != 8) return other_form();
        const at::Tensor *q = plain(a[0]), *k = plain(a[1]), *v = plain(a[2]), *o = plain(a[3]);
        Shape s;
        float scale, kscale, vscale;
        void* stream;
        if (!q || !k || !v || !o || !shape_of(*q, *k, *v, s) || o->sizes() != q->sizes()) return other_form();
        const int dt = dtype_of(*q);
        if (dt < 1 || o->scalar_type() != q->scalar_type() || k->scalar_type() != at::kFloat8_e4m3fn ||
            v->scalar_type() != at::kFloat8_e4m3fn)
            return other_form();
        const int causal = PyObject_IsTrue(a[4]);
        if (causal < 0 || !number(a[5], &scale) || !number(a[6], &kscale) || !number(a[7], &vscale) ||
            !current_stream(*q, &stream))
            return other_form();
        void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr(), *op = o->data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_attn_fwd_kv8(qp, kp, vp, op, s.B, s.Hq, s.Hkv, s.Lq, s.Lk, s.d, causal, scale, kscale, vscale, dt,
                            stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (...) {
        return other_form();
    }
}

// (q, k, v, causal, scale, o, state_in, state_out, causal_shift), the last four or None
PyObject* py_attn_fwd_state(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (n != 9) return other_form();
        const at::Tensor *q = plain(a[0]), *k = plain(a[1]), *v = plain(a[2]);
        const at::Tensor* out[3] = {nullptr, nullptr, nullptr};      // o, state_in, state_out
        Shape s;
        float scale;
        void* stream;
        if (!q || !k || !v || !shape_of(*q, *k, *v, s)) return other_form();
        const int dt = dtype_of(*q);
        if (dt < 0 || k->scalar_type() != q->scalar_type() || v->scalar_type() != q->scalar_type())
            return other_form();
        for (int i = 0; i < 3; ++i) {
            if (a[5 + i] == Py_None) continue;
            out[i] = plain(a[5 + i]);
            if (out[i] == nullptr) return other_form();
            const auto z = out[i]->sizes();
            if (z[0] != s.B || z[1] != s.Hq || z[2] != s.Lq || z[3] != s.d + (i > 0 ? 2 : 0) ||
                out[i]->scalar_type() != (i > 0 ? at::kFloat : q->scalar_type()))
                return other_form();
        }
        int shift = s.Lk - s.Lq;
        if (a[8] != Py_None) {
            const long x = PyLong_AsLong(a[8]);
            if ((x == -1 && PyErr_Occurred()) || x != (int)x) return other_form();
            shift = (int)x;
        }
        const int causal = PyObject_IsTrue(a[3]);
        if (causal < 0 || !number(a[4], &scale) || !current_stream(*q, &stream)) return other_form();
        void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
        void* op[3];
        for (int i = 0; i < 3; ++i) op[i] = out[i] ? out[i]->data_ptr() : nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_attn_fwd_state(qp, kp, vp, op[0], (const float*)op[1], (float*)op[2], s.B, s.Hq, s.Hkv, s.Lq, s.Lk,
                              s.d, causal, shift, scale, dt, stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (...) {
        return other_form();
    }
}

// ---- keys and values in pages ----------------------------------------------------------------------

decltype(&flashd_cache_fork) g_fork = nullptr;
decltype(&flashd_cache_reserve) g_reserve = nullptr;
decltype(&flashd_cache_append) g_append = nullptr;
decltype(&flashd_attn_fwd_tree) g_tree = nullptr;
decltype(&flashd_cache_commit) g_commit = nullptr;

// A plain GPU tensor of `dim` dimensions (0: any), or nullptr
const at::Tensor* on_gpu(PyObject* x, int dim) {
    if (!THPVariable_CheckExact(x)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(x);
    return t.is_cuda() && t.layout() == at::kStrided && (dim == 0 || t.dim() == dim) ? &t : nullptr;
}
// A contiguous one of whole numbers, on the device of `like` (nullptr: any); n: its size, -1: any
const at::Tensor* ints(PyObject* x, const at::Tensor* like, int64_t n = -1, int dim = 1) {
    const at::Tensor* t = on_gpu(x, dim);
    return t && t->scalar_type() == at::kInt && t->is_contiguous() && (!like || t->get_device() == like->get_device()) &&
                   (n < 0 || t->size(0) == n)
               ? t : nullptr;
}
bool small(int64_t n) { return n >= 1 && n <= 0x7fffffff; }

// The struct of a cache's tensors as flashd.py's _cache() makes it; false where that would refuse them
bool cache_of(PyObject* kx, PyObject* vx, PyObject* tx, PyObject* lx, bool layers, flashd_cache& c, const at::Tensor** kt) {
    const at::Tensor *k = on_gpu(kx, 0), *v = on_gpu(vx, 0);
    if (!k || !v || (k->dim() != 4 && !(layers && k->dim() == 5)) || k->sizes() != v->sizes() || k->strides() != v->strides() ||
        k->scalar_type() != v->scalar_type() || k->get_device() != v->get_device())
        return false;
    const int f = k->dim() - 4;
    const int64_t P = k->size(f), Hkv = k->size(f + 1), page = k->size(f + 2), d = k->size(f + 3);
    if (k->stride(f + 3) != 1 || k->stride(f + 2) != d || k->stride(f + 1) != page * d) return false;
    const at::Tensor* table = ints(tx, k, -1, 2);
    if (!table) return false;
    const int64_t B = table->size(0), cols = table->size(1);
    const at::Tensor* lens = ints(lx, k, B);
    if (!lens || !small(P) || !small(Hkv) || !small(page) || !small(d) || !small(B) || !small(cols) || (f && !small(k->size(0))))
        return false;
    const int dt = k->scalar_type() == at::kFloat8_e4m3fn ? FLASHD_CACHE_FP8 : dtype_of(*k);
    if (dt < 0) return false;
    c.k = k->data_ptr();
    c.v = v->data_ptr();
    c.table = static_cast<int*>(table->data_ptr());
    c.lens = static_cast<const int*>(lens->data_ptr());
    c.page_stride = P > 1 ? k->stride(f) : Hkv * page * d;
    c.layer_stride = f ? k->stride(0) : 0;
    c.layers = f ? (int)k->size(0) : 1;
    c.P = (int)P;
    c.page = (int)page;
    c.max_pages = (int)cols;
    c.B = (int)B;
    c.Hkv = (int)Hkv;
    c.d = (int)d;
    c.dtype = dt;
    c.kscale = c.vscale = 1.0f;
    *kt = k;
    return true;
}

// A packed tensor [T][heads][d] of type `like`'s and its stride; false where flashd.py would refuse it
bool packed(const at::Tensor* t, const at::Tensor& like, int64_t T, int64_t heads, int64_t d, long long* stride) {
    if (!t || t->get_device() != like.get_device() || t->scalar_type() != like.scalar_type() || t->size(0) != T ||
        t->size(1) != heads || t->size(2) != d || t->stride(2) != 1 || (heads > 1 && t->stride(1) != d))
        return false;
    *stride = T > 1 ? t->stride(0) : heads * d;
    return true;
}

template <typename F>
PyObject* call(F f) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// (parent, refs, table, lens, table_out, lens_out)
PyObject* py_cache_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (n != 6) return other_form();
        const at::Tensor* table = ints(a[2], nullptr, -1, 2);
        if (!table || !small(table->size(0)) || !small(table->size(1))) return other_form();
        const at::Tensor *parent = ints(a[0], table), *refs = ints(a[1], table), *lens = ints(a[3], table, table->size(0));
        if (!parent || !refs || !lens || !small(refs->size(0)) || !small(parent->size(0))) return other_form();
        const at::Tensor *tout = ints(a[4], table, parent->size(0), 2), *lout = ints(a[5], table, parent->size(0));
        void* stream;
        if (!tout || tout->size(1) != table->size(1) || !lout || !current_stream(*table, &stream)) return other_form();
        // (the pools themselves are not touched: any valid address and page size stand for them)
        const flashd_cache c{(void*)16, (void*)16, static_cast<int*>(table->data_ptr()), static_cast<const int*>(lens->data_ptr()),
                             16 * 64, 0, 1, (int)refs->size(0), 16, (int)table->size(1), (int)table->size(0), 1, 64, FLASHD_F16, 1.0f, 1.0f};
        int *rp = (int*)refs->data_ptr(), *pp = (int*)parent->data_ptr(), *to = (int*)tout->data_ptr(), *lo = (int*)lout->data_ptr();
        const int m = (int)parent->size(0);
        return call([&] { return g_fork(&c, rp, pp, m, to, lo, stream); });
    } catch (...) {
        return other_form();
    }
}

// (kcache, vcache, refs, table, lens, q_start, report)
PyObject* py_cache_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (n != 7) return other_form();
        flashd_cache c;
        const at::Tensor* k;
        void* stream;
        if (!cache_of(a[0], a[1], a[3], a[4], true, c, &k)) return other_form();
        const at::Tensor *refs = ints(a[2], k, c.P), *start = ints(a[5], k, c.B + 1LL), *report = ints(a[6], k, c.B + 1LL);
        if (!refs || !start || !report || !current_stream(*k, &stream)) return other_form();
        int *rp = (int*)refs->data_ptr(), *sp = (int*)start->data_ptr(), *out = (int*)report->data_ptr();
        return call([&] { return g_reserve(&c, rp, sp, out, stream); });
    } catch (...) {
        return other_form();
    }
}

// (kcache, vcache, table, lens, q_start, lens_out, keep, n_keep), the last two or None
PyObject* py_cache_commit(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (n != 8) return other_form();
        flashd_cache c;
        const at::Tensor *k, *keep = nullptr, *n_keep = nullptr;
        void* stream;
        if (!cache_of(a[0], a[1], a[2], a[3], true, c, &k)) return other_form();
        const at::Tensor *start = ints(a[4], k, c.B + 1LL), *out = ints(a[5], k, c.B);
        if (!start || !out) return other_form();
        if (a[6] != Py_None && (!(keep = ints(a[6], k, c.B, 2)) || !small(keep->size(1)))) return other_form();
        if (a[7] != Py_None && !(n_keep = ints(a[7], k, c.B))) return other_form();
        if (!current_stream(*k, &stream)) return other_form();
        int *sp = (int*)start->data_ptr(), *op = (int*)out->data_ptr(), *kp = keep ? (int*)keep->data_ptr() : nullptr,
            *np = n_keep ? (int*)n_keep->data_ptr() : nullptr;
        const int most = keep ? (int)keep->size(1) : 0;
        return call([&] { return g_commit(&c, sp, kp, most, np, op, stream); });
    } catch (...) {
        return other_form();
    }
}

// (q, k, v, q_out, kcache, vcache, table, lens, q_start, positions, inv_freq, q_weight, k_weight, eps, interleaved,
// kscale, vscale), the four after q_start or None
PyObject* py_cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (n != 17) return other_form();
        flashd_cache c;
        const at::Tensor* kc;
        void* stream;
        if (!cache_of(a[4], a[5], a[6], a[7], false, c, &kc)) return other_form();
        const at::Tensor *q = on_gpu(a[0], 3), *k = on_gpu(a[1], 3), *v = on_gpu(a[2], 3), *o = on_gpu(a[3], 3);
        if (!q || q->get_device() != kc->get_device()) return other_form();
        const int dt = dtype_of(*q);
        const int64_t T = q->size(0), Hq = q->size(1);
        long long s[4];
        if (dt < 0 || !small(T) || !small(Hq) || !packed(q, *q, T, Hq, c.d, s) || !packed(k, *q, T, c.Hkv, c.d, s + 1) ||
            !packed(v, *q, T, c.Hkv, c.d, s + 2) || !packed(o, *q, T, Hq, c.d, s + 3))
            return other_form();
        const at::Tensor *start = ints(a[8], kc, c.B + 1LL), *pos = nullptr, *inv = nullptr, *w[2] = {nullptr, nullptr};
        if (!start || (a[9] != Py_None && !(pos = ints(a[9], kc, T)))) return other_form();
        if (a[10] != Py_None) {
            inv = on_gpu(a[10], 1);
            if (!inv || inv->scalar_type() != at::kFloat || !inv->is_contiguous() || inv->get_device() != kc->get_device() ||
                inv->size(0) > 0xffff)
                return other_form();
        }
        for (int i = 0; i < 2; ++i) {
            if (a[11 + i] == Py_None) continue;
            w[i] = on_gpu(a[11 + i], 1);
            if (!w[i] || w[i]->scalar_type() != q->scalar_type() || !w[i]->is_contiguous() || w[i]->size(0) != c.d ||
                w[i]->get_device() != kc->get_device())
                return other_form();
        }
        float eps;
        const int inter = PyObject_IsTrue(a[14]);
        if (!number(a[13], &eps) || inter < 0 || !number(a[15], &c.kscale) || !number(a[16], &c.vscale) || !current_stream(*kc, &stream))
            return other_form();
        void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr(), *op = o->data_ptr();
        const int *sp = (const int*)start->data_ptr(), *pp = pos ? (const int*)pos->data_ptr() : nullptr;
        const float* ip = inv ? (const float*)inv->data_ptr() : nullptr;
        const void *w0 = w[0] ? w[0]->data_ptr() : nullptr, *w1 = w[1] ? w[1]->data_ptr() : nullptr;
        const int rot = inv ? 2 * (int)inv->size(0) : 0;
        return call([&] {
            return g_append(&c, 0, qp, s[0], kp, s[1], vp, s[2], op, s[3], (int)T, (int)Hq, sp, pp, ip, rot, inter, w0, w1, eps, dt, stream);
        });
    } catch (...) {
        return other_form();
    }
}

// (q, kcache, vcache, o, table, lens, q_start, max_q, scale, tree, kscale, vscale, workspace), tree and workspace or None
PyObject* py_attn_fwd_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (n != 13) return other_form();
        flashd_cache c;
        const at::Tensor* kc;
        void* stream;
        if (!cache_of(a[1], a[2], a[4], a[5], false, c, &kc)) return other_form();
        const at::Tensor *q = on_gpu(a[0], 3), *o = on_gpu(a[3], 3), *tree = nullptr, *ws = nullptr;
        if (!q || q->get_device() != kc->get_device()) return other_form();
        const int dt = dtype_of(*q);
        const int64_t T = q->size(0), Hq = q->size(1);
        long long s[2];
        if (dt < 0 || !small(T) || !small(Hq) || !packed(q, *q, T, Hq, c.d, s) || !packed(o, *q, T, Hq, c.d, s + 1)) return other_form();
        const at::Tensor* start = ints(a[6], kc, c.B + 1LL);
        const long max_q = PyLong_AsLong(a[7]);
        float scale;
        if (!start || (max_q == -1 && PyErr_Occurred()) || max_q != (int)max_q || !number(a[8], &scale)) return other_form();
        if (a[9] != Py_None) {
            tree = on_gpu(a[9], 2);
            if (!tree || tree->scalar_type() != at::kLong || !tree->is_contiguous() || tree->size(0) != T || !small(tree->size(1)) ||
                tree->get_device() != kc->get_device())
                return other_form();
        }
        if (a[12] != Py_None) {
            ws = on_gpu(a[12], 0);
            if (!ws || !ws->is_contiguous() || ws->get_device() != kc->get_device()) return other_form();
        }
        if (!number(a[10], &c.kscale) || !number(a[11], &c.vscale) || !current_stream(*kc, &stream)) return other_form();
        void *qp = q->data_ptr(), *op = o->data_ptr(), *wp = ws ? ws->data_ptr() : nullptr;
        const int* sp = (const int*)start->data_ptr();
        const unsigned long long* tp = tree ? (const unsigned long long*)tree->data_ptr() : nullptr;
        const size_t bytes = ws ? (size_t)ws->numel() * ws->element_size() : 0;
        const int words = tree ? (int)tree->size(1) : 0;
        return call([&] {
            return g_tree(&c, 0, qp, s[0], op, s[1], (int)T, (int)max_q, (int)Hq, sp, tp, words, scale, dt, stream, wp, bytes);
        });
    } catch (...) {
        return other_form();
    }
}

// (addresses of flashd_cache_fork, _reserve, _append, flashd_attn_fwd_tree, flashd_cache_commit)
PyObject* py_bind_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "bind_paged takes five addresses");
        return nullptr;
    }
    void* f[5];
    for (int i = 0; i < 5; ++i) f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    g_fork = reinterpret_cast<decltype(g_fork)>(f[0]);
    g_reserve = reinterpret_cast<decltype(g_reserve)>(f[1]);
    g_append = reinterpret_cast<decltype(g_append)>(f[2]);
    g_tree = reinterpret_cast<decltype(g_tree)>(f[3]);
    g_commit = reinterpret_cast<decltype(g_commit)>(f[4]);
    Py_RETURN_NONE;
}

// (address of flashd_attn_fwd, _kv8, _state, current-device function, raw-stream function)
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "bind takes three addresses and two functions");
        return nullptr;
    }
    void* f[3];
    for (int i = 0; i < 3; ++i) f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    g_attn_fwd = reinterpret_cast<attn_fwd_t>(f[0]);
    g_attn_fwd_kv8 = reinterpret_cast<attn_fwd_kv8_t>(f[1]);
    g_attn_fwd_state = reinterpret_cast<attn_fwd_state_t>(f[2]);
    Py_INCREF(a[3]);
    Py_XSETREF(g_current_device, a[3]);
    Py_INCREF(a[4]);
    Py_XSETREF(g_raw_stream, a[4]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_bind)), METH_FASTCALL, nullptr},
    {"attn_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_attn_fwd)), METH_FASTCALL, nullptr},
    {"attn_fwd_kv8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_attn_fwd_kv8)), METH_FASTCALL,
     nullptr},
    {"attn_fwd_state", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_attn_fwd_state)), METH_FASTCALL,
     nullptr},
    {"bind_paged", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_bind_paged)), METH_FASTCALL, nullptr},
    {"cache_fork", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_cache_fork)), METH_FASTCALL, nullptr},
    {"cache_reserve", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_cache_reserve)), METH_FASTCALL, nullptr},
    {"cache_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_cache_append)), METH_FASTCALL, nullptr},
    {"attn_fwd_tree", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_attn_fwd_tree)), METH_FASTCALL, nullptr},
    {"cache_commit", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_cache_commit)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_flashd_binding", nullptr, -1, methods, nullptr, nullptr, nullptr,
                      nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__flashd_binding() {
    PyObject* m = PyModule_Create(&module);
    // tensors are read through torch's C++ headers, so another version's may not be handed in
    // (FLASHD_TORCH: torch.__version__ at the build)
    const char* built_for =
        "torch " FLASHD_TORCH " and Python " Py_STRINGIFY(PY_MAJOR_VERSION) "." Py_STRINGIFY(PY_MINOR_VERSION);
    if (m != nullptr && PyModule_AddStringConstant(m, "built_for", built_for) != 0) Py_CLEAR(m);
    return m;
}
