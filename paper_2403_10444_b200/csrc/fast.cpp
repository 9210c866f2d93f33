// The binding's calls of the paged cache in C++ (module _fast): the checks of binding.py on tensors of the ordinary kind, the library's call, and
// nothing else.  A call of the cache takes some 5 us of GPU and driver time, and marshalling it in the interpreter another 7.
// What is out of the ordinary (a tensor of the wrong type or shape, an empty batch, an output with gaps, another device than the current one) is
// left to binding.py: NotImplemented.  A status that is not 0 comes back as an integer, for binding.py to raise.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <exception>

#include "../../include/bv.h"

namespace {

decltype(&bv_cache_attend) f_attend = nullptr;
decltype(&bv_cache_append) f_append = nullptr;
decltype(&bv_pages_extend) f_extend = nullptr;
decltype(&bv_pages_truncate) f_truncate = nullptr;
decltype(&bv_pages_fork) f_fork = nullptr;
decltype(&bv_pages_compact) f_compact = nullptr;
decltype(&bv_pages_copy) f_copy = nullptr;

PyObject* other() { Py_RETURN_NOTIMPLEMENTED; }
const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
template <typename T> T* address(const at::Tensor& t) { return static_cast<T*>(t.data_ptr()); }

// torch's current stream on `dev`; false if another device is current.
bool stream_of(int dev, void** s) {
    if (c10::cuda::current_device() != dev) return false;
    *s = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(dev)).stream();
    return true;
}
// A contiguous int32 [n] on `dev`, or None if that may be.
bool counted(PyObject* o, int64_t n, int dev, bool none, int32_t** p) {
    *p = nullptr;
    if (o == Py_None) return none;
    const at::Tensor* t = tensor(o);
    if (!t || t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != n || !t->is_contiguous() || !t->is_cuda() || t->get_device() != dev) return false;
    *p = address<int32_t>(*t);
    return true;
}
bool sequences(PyObject* table, PyObject* lens, bv_cache* c, int* dev) {
    const at::Tensor *t = tensor(table), *l = tensor(lens);
    if (!t || !l || t->scalar_type() != at::kInt || l->scalar_type() != at::kInt || t->dim() != 2 || l->dim() != 1 || l->size(0) != t->size(0) || !t->is_contiguous() ||
        !l->is_contiguous() || !t->is_cuda() || !l->is_cuda() || l->get_device() != t->get_device()) return false;
    if (t->size(0) > INT32_MAX || t->size(1) > INT32_MAX || t->size(0) == 0) return false;
    *dev = static_cast<int>(t->get_device());
    c->table = address<int32_t>(*t);
    c->lens = address<int32_t>(*l);
    c->B = static_cast<int32_t>(t->size(0));
    c->width = static_cast<int32_t>(t->size(1));
    return true;
}
// Two pools of pages [num_pages, heads, page_size, D] of one shape; `written`: contiguous ones (no two elements in one place).
bool pools(const at::Tensor* k, const at::Tensor* v, bool written, bv_cache* c, int* dev) {
    if (!k || !v || k->dim() != 4 || v->dim() != 4 || k->sizes() != v->sizes() || k->scalar_type() != v->scalar_type() || !k->is_cuda() || !v->is_cuda() ||
        k->get_device() != v->get_device() || k->stride(3) != 1 || v->stride(3) != 1) return false;
    if (k->scalar_type() == at::kFloat) c->dtype = BV_DTYPE_F32;
    else if (k->scalar_type() == at::kBFloat16) c->dtype = BV_DTYPE_BF16;
    else return false;
    if (written && !(k->is_contiguous() && v->is_contiguous())) return false;
    for (int i = 0; i < 4; ++i)
        if (k->size(i) > INT32_MAX) return false;
    c->k = k->data_ptr();
    c->v = v->data_ptr();
    for (int i = 0; i < 3; ++i) {
        c->k_stride[i] = k->stride(i);
        c->v_stride[i] = v->stride(i);
    }
    c->num_pages = static_cast<int32_t>(k->size(0));
    c->heads = static_cast<int32_t>(k->size(1));
    c->page_size = static_cast<int32_t>(k->size(2));
    c->D = static_cast<int32_t>(k->size(3));
    *dev = static_cast<int>(k->get_device());
    return true;
}
// [B, n, heads, D] that goes with the cache (heads = 0: any number).
bool rows(const at::Tensor* t, const bv_cache& c, const at::Tensor& k, int64_t heads, int dev, int64_t* stride) {
    if (!t || t->dim() != 4 || t->size(0) != c.B || t->size(3) != c.D || (heads && t->size(2) != heads) || t->scalar_type() != k.scalar_type() || !t->is_cuda() ||
        t->get_device() != dev || t->stride(3) != 1 || t->size(1) > INT32_MAX || t->size(2) > INT32_MAX) return false;
    for (int i = 0; i < 3; ++i) stride[i] = t->stride(i);
    return true;
}
// An integer of 32 bits.
bool whole(PyObject* o, int* x) {
    if (!PyLong_Check(o)) return false;
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    if (over != 0 || v > INT32_MAX || v < INT32_MIN) return false;
    *x = static_cast<int>(v);
    return true;
}
bool book(PyObject* table, PyObject* lens, PyObject* refs, PyObject* page, bv_cache* c, int* dev) {
    if (!sequences(table, lens, c, dev)) return false;
    const at::Tensor* r = tensor(refs);
    if (!r || r->scalar_type() != at::kInt || r->dim() != 1 || !r->is_contiguous() || !r->is_cuda() || r->get_device() != *dev || r->size(0) > INT32_MAX) return false;
    int p;
    if (!whole(page, &p)) return false;
    c->refs = address<int32_t>(*r);
    c->num_pages = static_cast<int32_t>(r->size(0));
    c->page_size = p;
    return true;
}
// The answer: `result` (a new reference) or the status.
PyObject* answer(int status, PyObject* result) {
    if (status == 0) return result;
    Py_XDECREF(result);
    return PyLong_FromLong(status);
}
PyObject* none() { return Py_NewRef(Py_None); }

// (Exceptions of torch end here: what it would not do, binding.py tries again and reports.)
template <typename F> PyObject* guarded(F f) {
    try {
        return f();
    } catch (const std::exception&) {
        return other();
    }
}
template <typename F> int released(F f) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    return status;
}

// q, k, v, table, lens, n_new, scale, window, sinks, out
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 10 || !f_attend) return other();
    return guarded([&]() -> PyObject* {
        bv_cache c{};
        int dev, at, window, sinks;
        void* s;
        int32_t* n_new;
        int64_t qs[3], os[3];
        const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *v = tensor(a[2]);
        if (!pools(k, v, false, &c, &dev) || !sequences(a[3], a[4], &c, &at) || at != dev || !rows(q, c, *k, 0, dev, qs) || !counted(a[5], c.B, dev, true, &n_new) ||
            !whole(a[7], &window) || !whole(a[8], &sinks) || !stream_of(dev, &s)) return other();
        double scale = 1.0 / std::sqrt(static_cast<double>(c.D));
        if (a[6] != Py_None) {
            if (!PyFloat_Check(a[6])) return other();
            scale = PyFloat_AS_DOUBLE(a[6]);
        }
        at::Tensor made;
        const at::Tensor* out;
        if (a[9] == Py_None) {
            made = n_new ? at::zeros(q->sizes(), q->options().requires_grad(false)) : at::empty(q->sizes(), q->options().requires_grad(false));
            out = &made;
        } else {
            out = tensor(a[9]);
            if (!out || !out->is_contiguous()) return other();
        }
        if (!rows(out, c, *k, q->size(2), dev, os) || out->size(1) != q->size(1)) return other();
        const int status = released([&] {
            return f_attend(&c, q->data_ptr(), qs, n_new, static_cast<int>(q->size(1)), static_cast<int>(q->size(2)), static_cast<float>(scale), window, sinks, out->data_ptr(), os, s);
        });
        if (status != 0) return PyLong_FromLong(status);
        return a[9] == Py_None ? THPVariable_Wrap(made) : Py_NewRef(a[9]);
    });
}
// k_new, v_new, k, v, table, lens, n_new
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7 || !f_append) return other();
    return guarded([&]() -> PyObject* {
        bv_cache c{};
        int dev, at;
        void* s;
        int32_t* n_new;
        int64_t ks[3], vs[3];
        const at::Tensor *kn = tensor(a[0]), *vn = tensor(a[1]), *k = tensor(a[2]), *v = tensor(a[3]);
        if (!pools(k, v, true, &c, &dev) || !sequences(a[4], a[5], &c, &at) || at != dev || !rows(kn, c, *k, c.heads, dev, ks) || !rows(vn, c, *k, c.heads, dev, vs) ||
            vn->size(1) != kn->size(1) || !counted(a[6], c.B, dev, true, &n_new) || !stream_of(dev, &s)) return other();
        return answer(released([&] { return f_append(&c, kn->data_ptr(), ks, vn->data_ptr(), vs, n_new, static_cast<int>(kn->size(1)), s); }), none());
    });
}
// table, lens, refs, page_size, n, n_new
PyObject* extend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6 || !f_extend) return other();
    return guarded([&]() -> PyObject* {
        bv_cache c{};
        int dev, most;
        void* s;
        int32_t* n_new;
        if (!book(a[0], a[1], a[2], a[3], &c, &dev) || !whole(a[4], &most) || !counted(a[5], c.B, dev, true, &n_new) || !stream_of(dev, &s)) return other();
        const auto options = tensor(a[0])->options();
        const at::Tensor got = at::empty({c.B}, options), copies = at::empty({c.B, 2}, options);
        const int status = released([&] { return f_extend(&c, n_new, most, address<int32_t>(got), address<int32_t>(copies), s); });
        if (status != 0) return PyLong_FromLong(status);
        PyObject* both = PyTuple_New(2);
        if (!both) return nullptr;
        PyTuple_SET_ITEM(both, 0, THPVariable_Wrap(got));
        PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(copies));
        return both;
    });
}
// table, lens, refs, page_size, keep, n, n_new
PyObject* truncate(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7 || !f_truncate) return other();
    return guarded([&]() -> PyObject* {
        bv_cache c{};
        int dev, most;
        void* s;
        int32_t *keep, *n_new;
        if (!book(a[0], a[1], a[2], a[3], &c, &dev) || !counted(a[4], c.B, dev, false, &keep) || !whole(a[5], &most) || !counted(a[6], c.B, dev, true, &n_new) ||
            !stream_of(dev, &s)) return other();
        return answer(released([&] { return f_truncate(&c, keep, n_new, most, s); }), none());
    });
}
// table, lens, refs, page_size, src, dst
PyObject* fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6 || !f_fork) return other();
    return guarded([&]() -> PyObject* {
        bv_cache c{};
        int dev;
        void* s;
        int32_t *src, *dst;
        const at::Tensor* first = tensor(a[4]);
        if (!first || first->dim() != 1 || first->size(0) < 1 || first->size(0) > INT32_MAX) return other();
        const int forks = static_cast<int>(first->size(0));
        if (!book(a[0], a[1], a[2], a[3], &c, &dev) || !counted(a[4], forks, dev, false, &src) || !counted(a[5], forks, dev, false, &dst) || !stream_of(dev, &s)) return other();
        const at::Tensor ok = at::empty({forks}, tensor(a[0])->options());
        const int status = released([&] { return f_fork(&c, src, dst, forks, address<int32_t>(ok), s); });
        return status ? PyLong_FromLong(status) : THPVariable_Wrap(ok);
    });
}
// table, lens, refs, page_size
PyObject* compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4 || !f_compact) return other();
    return guarded([&]() -> PyObject* {
        bv_cache c{};
        int dev;
        void* s;
        if (!book(a[0], a[1], a[2], a[3], &c, &dev) || c.num_pages < 2 || !stream_of(dev, &s)) return other();
        const auto options = tensor(a[0])->options();
        const at::Tensor moves = at::empty({c.num_pages / 2, 2}, options), count = at::empty({1}, options);
        const int status = released([&] { return f_compact(&c, address<int32_t>(moves), address<int32_t>(count), s); });
        if (status != 0) return PyLong_FromLong(status);
        PyObject* both = PyTuple_New(2);
        if (!both) return nullptr;
        PyTuple_SET_ITEM(both, 0, THPVariable_Wrap(moves));
        PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(count));
        return both;
    });
}
// k, v, pairs, count
PyObject* copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4 || !f_copy) return other();
    return guarded([&]() -> PyObject* {
        bv_cache c{};
        int dev;
        void* s;
        int32_t* count;
        const at::Tensor* pairs = tensor(a[2]);
        if (!pools(tensor(a[0]), tensor(a[1]), true, &c, &dev) || !pairs || pairs->scalar_type() != at::kInt || pairs->dim() != 2 || pairs->size(1) != 2 || pairs->size(0) < 1 ||
            pairs->size(0) > INT32_MAX || !pairs->is_contiguous() || !pairs->is_cuda() || pairs->get_device() != dev || !counted(a[3], 1, dev, true, &count) || !stream_of(dev, &s))
            return other();
        return answer(released([&] { return f_copy(&c, address<int32_t>(*pairs), static_cast<int>(pairs->size(0)), count, s); }), none());
    });
}
// The addresses of the library's entry points, in the order of the functions above.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[7];
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "bind takes seven addresses");
        return nullptr;
    }
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    f_attend = reinterpret_cast<decltype(f_attend)>(p[0]);
    f_append = reinterpret_cast<decltype(f_append)>(p[1]);
    f_extend = reinterpret_cast<decltype(f_extend)>(p[2]);
    f_truncate = reinterpret_cast<decltype(f_truncate)>(p[3]);
    f_fork = reinterpret_cast<decltype(f_fork)>(p[4]);
    f_compact = reinterpret_cast<decltype(f_compact)>(p[5]);
    f_copy = reinterpret_cast<decltype(f_copy)>(p[6]);
    return none();
}

#define BV_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {BV_METHOD(attend), BV_METHOD(append), BV_METHOD(extend), BV_METHOD(truncate), BV_METHOD(fork), BV_METHOD(compact), BV_METHOD(copy), BV_METHOD(bind),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_fast", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit__fast() { return PyModule_Create(&module_def); }
