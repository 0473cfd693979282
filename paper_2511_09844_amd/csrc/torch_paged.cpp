// The paged calls on torch tensors that are as they should be (paged.py): the checks, the arguments and the call in one
// step, 0.5 us of host time where Python takes 5 to 9 beside the launch.  Any argument that is not a plain case of what
// the call documents, and any refusal (SD2_ERR_INVALID_ARG, which comes before anything is enqueued), gives None, and
// paged.py's own checks say what is wrong.  A call that failed otherwise is not to be made again, as it may have enqueued a
// part of its work (sd2_pages_reserve: the tables, but not the copies that they ask for): its error is raised here.
//
// These calls are bound by the host otherwise: one row of each of 16 sequences is appended in 4.4 us on the GPU.
#include <Python.h>

#include <vector>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/sd2.h"

namespace {

struct Cache {
    int device, n_layers, hd, hkv, max_seqs, max_pages, page_size;
    bool held8;                            // scaled
    bool takes[2];                         // rows of fp32, of bf16
    std::vector<sd2_paged_kv> kv[2];       // by the rows' dtype, a layer each
    std::vector<sd2_paged_scaled> scaled[2];
    sd2_pages pages;
    void* unused;                          // workspace of calls that need none
    size_t pages_ws;
    float scale;
};

const char* const kName = "paged cache";
Cache* cache_of(PyObject* o) { return static_cast<Cache*>(PyCapsule_GetPointer(o, kName)); }

bool int_of(PyObject* o, int64_t lo, int64_t hi, int64_t& v) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    v = PyLong_AsLongLongAndOverflow(o, &over);
    return !over && v >= lo && v <= hi;
}

const at::Tensor* tensor_of(PyObject* o, const Cache& c) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.layout() == at::kStrided && t.is_cuda() && t.get_device() == c.device ? &t : nullptr;
}

const at::Tensor* int32_of(PyObject* o, const Cache& c) {
    const at::Tensor* t = tensor_of(o, c);
    return t && t->scalar_type() == at::kInt && t->dim() == 1 && t->is_contiguous() ? t : nullptr;
}

// Rows [rows][heads][head_dim], their type (0: fp32, 1: bf16) and row stride.
struct Packed {
    const at::Tensor* t = nullptr;
    int dtype = -1;
    int64_t stride = 0;
};
bool packed_of(PyObject* o, const Cache& c, Packed& p) {
    p.t = tensor_of(o, c);
    if (!p.t || p.t->dim() != 3 || p.t->size(2) != c.hd || (p.t->requires_grad() && c10::GradMode::is_enabled())) return false;
    p.dtype = p.t->scalar_type() == at::kFloat ? 0 : p.t->scalar_type() == at::kBFloat16 ? 1 : -1;
    if (p.dtype < 0 || !c.takes[p.dtype]) return false;
    if (p.t->numel() && (p.t->stride(2) != 1 || (p.t->size(1) != 1 && p.t->stride(1) != c.hd))) return false;
    p.stride = p.t->size(0) > 1 ? p.t->stride(0) : p.t->size(1) * c.hd;
    return true;
}

bool rows_of(int64_t total, PyObject* lens, PyObject* row_off, PyObject* max_rows, const Cache& c, sd2_paged_rows& r) {
    const at::Tensor* l = int32_of(lens, c);
    if (!l || l->numel() > c.max_seqs || total > INT32_MAX) return false;
    const int64_t n = l->numel();
    int64_t most = 0;
    if (max_rows != Py_None && !int_of(max_rows, 0, INT32_MAX, most)) return false;
    r.lens = static_cast<const int32_t*>(l->data_ptr());
    if (row_off == Py_None) {
        if (n ? total % n != 0 : total != 0) return false;
        const int64_t each = n ? total / n : 0;
        if (max_rows != Py_None && most != each) return false;
        r.nseq = each ? n : 0;
        r.max_rows = each ? each : 1;
        r.total_rows = n ? total : 0;
        r.row_off = nullptr;
        return true;
    }
    const at::Tensor* off = int32_of(row_off, c);
    if (!off || off->numel() != n + 1 || (max_rows != Py_None && most < 1)) return false;
    r.nseq = n;
    r.max_rows = max_rows != Py_None ? most : total > 1 ? total : 1;
    r.total_rows = total;
    r.row_off = static_cast<const int32_t*>(off->data_ptr());
    return true;
}

// A call without the interpreter's lock.
template <typename F>
sd2_status unlocked(F f) {
    PyThreadState* s = PyEval_SaveThread();
    const sd2_status rc = f();
    PyEval_RestoreThread(s);
    return rc;
}

at::Tensor bytes(size_t n, const at::Tensor& like) {
    return at::empty({(int64_t)n}, like.options().dtype(at::kByte));
}

#define NONE_IF(cond) \
    if (cond) Py_RETURN_NONE

// What a call that was made gives: result (a new reference, made before the call: nothing may throw behind it), None where it
// was refused, else the exception that binding.check makes of its status.
PyObject* ended(sd2_status rc, const char* call, PyObject* result) {
    if (rc == SD2_OK) return result;
    Py_DECREF(result);
    NONE_IF(rc == SD2_ERR_INVALID_ARG);
    if (PyObject* binding = PyImport_ImportModule("paper_2511_09844_amd.binding")) {
        Py_XDECREF(PyObject_CallMethod(binding, "check", "iOs", (int)rc, Py_None, call));
        Py_DECREF(binding);
    }
    if (!PyErr_Occurred()) PyErr_Format(PyExc_RuntimeError, "%s: status %d", call, (int)rc);
    return nullptr;
}
PyObject* new_true() {
    Py_INCREF(Py_True);
    return Py_True;
}

// cache(device, n_layers, hd, hkv, max_seqs, max_pages, page_size, held8, kv of fp32 rows, of bf16 rows (addresses or 0),
// pages (address), unused workspace, workspace bytes of pages, scale)
PyObject* make_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 14) return PyErr_Format(PyExc_TypeError, "cache: 14 arguments");
    int64_t v[13];
    for (int i = 0; i < 13; ++i) {
        v[i] = PyLong_AsLongLong(a[i]);
        if (v[i] == -1 && PyErr_Occurred()) return nullptr;
    }
    const double scale = PyFloat_AsDouble(a[13]);
    if (scale == -1.0 && PyErr_Occurred()) return nullptr;
    Cache* c = new Cache{};
    c->device = v[0]; c->n_layers = v[1]; c->hd = v[2]; c->hkv = v[3]; c->max_seqs = v[4]; c->max_pages = v[5]; c->page_size = v[6];
    c->held8 = v[7];
    for (int t = 0; t < 2; ++t) {
        c->takes[t] = v[8 + t] != 0;
        if (!c->takes[t]) continue;
        if (c->held8) {
            const sd2_paged_scaled* p = reinterpret_cast<const sd2_paged_scaled*>(v[8 + t]);
            c->scaled[t].assign(p, p + c->n_layers);
        } else {
            const sd2_paged_kv* p = reinterpret_cast<const sd2_paged_kv*>(v[8 + t]);
            c->kv[t].assign(p, p + c->n_layers);
        }
    }
    c->pages = *reinterpret_cast<const sd2_pages*>(v[10]);
    c->unused = reinterpret_cast<void*>(v[11]);
    c->pages_ws = v[12];
    c->scale = scale;
    return PyCapsule_New(c, kName, [](PyObject* o) { delete cache_of(o); });
}

// append(cache, stream, k, v, lens, layer, row_off, max_rows): True, or None
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 8) return PyErr_Format(PyExc_TypeError, "append: 8 arguments");
    Cache* c = cache_of(a[0]);
    if (!c) return nullptr;
    int64_t stream, layer;
    Packed k, v;
    sd2_paged_rows r;
    NONE_IF(!int_of(a[1], 0, INT64_MAX, stream) || !packed_of(a[2], *c, k) || !packed_of(a[3], *c, v) || k.dtype != v.dtype);
    NONE_IF(k.t->sizes() != v.t->sizes() || k.t->size(1) != c->hkv || !int_of(a[5], 0, c->n_layers - 1, layer));
    NONE_IF(!rows_of(k.t->size(0), a[4], a[6], a[7], *c, r));
    const void *kp = k.t->data_ptr(), *vp = v.t->data_ptr();
    const sd2_status rc = unlocked([&] {
        return c->held8 ? sd2_paged_append_scaled(&c->scaled[k.dtype][layer], &r, kp, k.stride, vp, v.stride, reinterpret_cast<void*>(stream))
                        : sd2_paged_append(&c->kv[k.dtype][layer], &r, kp, k.stride, vp, v.stride, reinterpret_cast<void*>(stream));
    });
    return ended(rc, c->held8 ? "sd2_paged_append_scaled" : "sd2_paged_append", new_true());
}

// attend(cache, stream, q, lens, layer, row_off, max_rows, max_len, scale, out, window, sinks): out, or None
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 12) return PyErr_Format(PyExc_TypeError, "attend: 12 arguments");
    Cache* c = cache_of(a[0]);
    if (!c) return nullptr;
    int64_t stream, layer, max_len = (int64_t)c->max_pages * c->page_size, window = 0, sinks;
    Packed q, o;
    sd2_paged_rows r;
    NONE_IF(!int_of(a[1], 0, INT64_MAX, stream) || !packed_of(a[2], *c, q) || !int_of(a[4], 0, c->n_layers - 1, layer));
    const int64_t heads = q.t->size(1);
    NONE_IF(heads < 1 || heads % c->hkv || !rows_of(q.t->size(0), a[3], a[5], a[6], *c, r));
    NONE_IF(a[7] != Py_None && !int_of(a[7], 1, max_len, max_len));
    NONE_IF(a[8] != Py_None && !PyFloat_CheckExact(a[8]));
    const float scale = a[8] == Py_None ? c->scale : (float)PyFloat_AS_DOUBLE(a[8]);
    NONE_IF(a[10] != Py_None && !int_of(a[10], 1, 1 << 30, window));
    NONE_IF(!int_of(a[11], 0, window ? 1 << 30 : 0, sinks));
    at::Tensor out, ws;
    if (a[9] == Py_None) {
        out = at::empty(q.t->sizes(), q.t->options());
        o.stride = heads * c->hd;
    } else {
        NONE_IF(!packed_of(a[9], *c, o) || o.dtype != q.dtype || o.t->sizes() != q.t->sizes());
        NONE_IF(q.t->numel() && o.t->data_ptr() == q.t->data_ptr());
        out = *o.t;
    }
    const sd2_paged_kv* kv = c->held8 ? nullptr : &c->kv[q.dtype][layer];
    const sd2_paged_scaled* sc = c->held8 ? &c->scaled[q.dtype][layer] : nullptr;
    const size_t need = sc ? sd2_paged_attn_scaled_workspace_bytes(sc, &r, heads, max_len, window, sinks)
                           : sd2_paged_attn_window_workspace_bytes(kv, &r, heads, max_len, window, sinks);
    NONE_IF(!need);
    void* w = c->unused;
    if (need > 256) {
        ws = bytes(need, *q.t);
        w = ws.data_ptr();
    }
    const void* qp = q.t->data_ptr();
    void* op = out.data_ptr();
    PyObject* result = a[9];
    if (result == Py_None) result = THPVariable_Wrap(std::move(out));
    else Py_INCREF(result);
    if (!result) return nullptr;
    const sd2_status rc = unlocked([&] {
        return sc ? sd2_paged_attn_scaled(sc, &r, qp, q.stride, op, o.stride, heads, scale, max_len, window, sinks, w, need, reinterpret_cast<void*>(stream))
                  : sd2_paged_attn_window(kv, &r, qp, q.stride, op, o.stride, heads, scale, max_len, window, sinks, w, need, reinterpret_cast<void*>(stream));
    });
    return ended(rc, sc ? "sd2_paged_attn_scaled" : window ? "sd2_paged_attn_window" : "sd2_paged_attn", result);
}

// A list, tuple or range of sequences of the table.
bool seqs_of(PyObject* o, const Cache& c, std::vector<int32_t>& v) {
    if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o) && !PyRange_Check(o)) return false;
    PyObject* f = PySequence_Fast(o, "");
    if (!f) {
        PyErr_Clear();
        return false;
    }
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(f);
    v.resize(n);
    bool ok = n <= c.max_seqs;
    for (Py_ssize_t i = 0; ok && i < n; ++i) {
        int64_t x = 0;
        ok = int_of(PySequence_Fast_GET_ITEM(f, i), 0, c.max_seqs - 1, x);
        v[i] = x;
    }
    Py_DECREF(f);
    return ok;
}

// fork(cache, stream, src, dst): True, or None
PyObject* fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4) return PyErr_Format(PyExc_TypeError, "fork: 4 arguments");
    Cache* c = cache_of(a[0]);
    if (!c) return nullptr;
    int64_t stream;
    std::vector<int32_t> src, dst;
    NONE_IF(!int_of(a[1], 0, INT64_MAX, stream) || !seqs_of(a[2], *c, src) || !seqs_of(a[3], *c, dst) || src.size() != dst.size() || src.empty());
    const sd2_status rc = unlocked([&] { return sd2_pages_fork(&c->pages, src.size(), src.data(), dst.data(), reinterpret_cast<void*>(stream)); });
    return ended(rc, "sd2_pages_fork", new_true());
}

// slide(cache, stream, lens, window, sinks): True, or None
PyObject* slide(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) return PyErr_Format(PyExc_TypeError, "slide: 5 arguments");
    Cache* c = cache_of(a[0]);
    if (!c) return nullptr;
    int64_t stream, window, sinks;
    const at::Tensor* lens = int32_of(a[2], *c);
    NONE_IF(!int_of(a[1], 0, INT64_MAX, stream) || !lens || lens->numel() > c->max_seqs);
    NONE_IF(!int_of(a[3], 1, 1 << 30, window) || !int_of(a[4], 0, 1 << 30, sinks));
    const int32_t* p = static_cast<const int32_t*>(lens->data_ptr());
    const int32_t m = lens->numel();
    const sd2_status rc = unlocked([&] { return sd2_pages_slide(&c->pages, m, p, window, sinks, reinterpret_cast<void*>(stream)); });
    return ended(rc, "sd2_pages_slide", new_true());
}

// reserve(cache, stream, first, last, keep): granted, or None
PyObject* reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) return PyErr_Format(PyExc_TypeError, "reserve: 5 arguments");
    Cache* c = cache_of(a[0]);
    if (!c) return nullptr;
    int64_t stream;
    const at::Tensor *first = int32_of(a[2], *c), *last = int32_of(a[3], *c), *keep = a[4] == Py_None ? nullptr : int32_of(a[4], *c);
    NONE_IF(!int_of(a[1], 0, INT64_MAX, stream) || !first || !last || (a[4] != Py_None && !keep));
    const int64_t m = first->numel();
    NONE_IF(last->numel() != m || (keep && keep->numel() != m) || m > c->max_seqs);
    at::Tensor granted = at::empty(last->sizes(), last->options()), ws = bytes(c->pages_ws, *last);
    auto ints = [](const at::Tensor* t) { return t ? static_cast<const int32_t*>(t->data_ptr()) : nullptr; };
    const int32_t *f = ints(first), *l = ints(last), *k = ints(keep);
    int32_t* g = static_cast<int32_t*>(granted.data_ptr());
    void* w = ws.data_ptr();
    PyObject* result = THPVariable_Wrap(std::move(granted));
    if (!result) return nullptr;
    const sd2_status rc = unlocked([&] { return sd2_pages_reserve(&c->pages, m, f, l, k, g, w, c->pages_ws, reinterpret_cast<void*>(stream)); });
    return ended(rc, "sd2_pages_reserve", result);
}

// What torch throws (an allocation that fails, say: all of it before the library's call) comes again, as its own exception, from
// the call that paged.py makes then.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    try {
        return F(self, a, n);
    } catch (const std::exception&) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

#define METHOD(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<fn>)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {METHOD("cache", make_cache), METHOD("append", append), METHOD("attend", attend), METHOD("fork", fork),
                          METHOD("slide", slide), METHOD("reserve", reserve), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_torch_paged", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_paged() { return PyModule_Create(&kModule); }
