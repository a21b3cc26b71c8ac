// Python module that hands torch tensors to the key/value store calls of the C ABI: it checks types, shapes, devices and
// strides and makes the call, all in one step. (Through ctypes the same checks and conversions took 7 to 8 us a call, more than
// most decode-sized kernels run; here they take well under one.) It holds no state but the addresses of the library's functions,
// so that it serves every build of the library.
#include <Python.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "gkv.h"

namespace {

decltype(&gkv_store_write) g_write;
decltype(&gkv_store_read) g_read;
decltype(&gkv_store_attn) g_attn;

const char* type_name(at::ScalarType t) { return c10::toString(t); }

const at::Tensor* tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_ValueError, "%s: a tensor is needed, got %s", what, Py_TYPE(o)->tp_name);
        return nullptr;
    }
    return &THPVariable_Unpack(o);
}
bool refuse(const char* what, at::ScalarType type, at::IntArrayRef shape, int device, const at::Tensor& t) {
    std::ostringstream s;
    s << what << ": a contiguous " << type_name(type) << " tensor of shape " << shape << " on cuda:" << device << " is needed, got "
      << type_name(t.scalar_type()) << " " << t.sizes() << " on " << t.device() << (t.is_contiguous() ? "" : ", not contiguous");
    PyErr_SetString(PyExc_ValueError, s.str().c_str());
    return false;
}
// Data pointer of a contiguous tensor of this type, shape and device; None gives NULL where that is allowed.
bool pointer(PyObject* o, const char* what, at::ScalarType type, at::IntArrayRef shape, int device, bool optional, void** out) {
    *out = nullptr;
    if (optional && o == Py_None) return true;
    const at::Tensor* t = tensor(o, what);
    if (!t) return false;
    if (t->scalar_type() != type || t->sizes() != shape || !t->is_cuda() || t->get_device() != device || !t->is_contiguous())
        return refuse(what, type, shape, device, *t);
    *out = t->data_ptr();
    return true;
}
bool current_stream(int device, void** stream) {
    const int current = c10::cuda::current_device();
    if (current != device) {
        PyErr_Format(PyExc_ValueError, "the store is on cuda:%d, the current device is cuda:%d", device, current);
        return false;
    }
    *stream = c10::cuda::getCurrentCUDAStream(device).stream();
    return true;
}
bool arguments(Py_ssize_t n, Py_ssize_t want, const char* what) {
    if (n != want) PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", what, want, n);
    return n == want;
}
template <typename T>
T* address(PyObject* o) { return reinterpret_cast<T*>(PyLong_AsUnsignedLongLong(o)); }

// bind(write, read, attn): addresses of the library's functions
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arguments(n, 3, "bind")) return nullptr;
    g_write = reinterpret_cast<decltype(g_write)>(PyLong_AsUnsignedLongLong(a[0]));
    g_read = reinterpret_cast<decltype(g_read)>(PyLong_AsUnsignedLongLong(a[1]));
    g_attn = reinterpret_cast<decltype(g_attn)>(PyLong_AsUnsignedLongLong(a[2]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

// copy(read, store, device, k, v, first, count) -> status
PyObject* copy(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    if (!arguments(n, 7, "copy")) return nullptr;
    const bool read = a[0] == Py_True;
    const gkv_store* s = address<const gkv_store>(a[1]);
    const int device = (int)PyLong_AsLong(a[2]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *k = tensor(a[3], "k"), *v = k ? tensor(a[4], "v") : nullptr;
    if (!v) return nullptr;
    int64_t strides[3] = {0, 0, 0};
    for (const at::Tensor* t : {k, v}) {
        if (t->scalar_type() != at::kBFloat16 || t->dim() != 4 || t->size(0) != s->batch || t->size(2) != s->n_kv_heads ||
            t->size(3) != s->head_dim || t->sizes() != k->sizes() || !t->is_cuda() || t->get_device() != device) {
            std::ostringstream m;
            m << (t == k ? "k" : "v") << ": a BFloat16 tensor [" << s->batch << "][tokens][" << s->n_kv_heads << "][" << s->head_dim
              << "] on cuda:" << device << " is needed, got " << type_name(t->scalar_type()) << " " << t->sizes() << " on " << t->device();
            PyErr_SetString(PyExc_ValueError, m.str().c_str());
            return nullptr;
        }
        bool fine = t->stride(3) == 1;
        for (int i = 0; i < 3; ++i) {           // strides of steps that are taken
            const int64_t st = t->size(i) == 1 ? 0 : t->stride(i);
            if (t == k) strides[i] = st;
            else fine = fine && st == strides[i];
        }
        if (!fine) {
            std::ostringstream m;
            m << "k, v: strides " << k->strides() << ", " << v->strides() << ": the last one has to be 1, and the two have to agree";
            PyErr_SetString(PyExc_ValueError, m.str().c_str());
            return nullptr;
        }
    }
    void *first, *count, *stream;
    const int64_t batch[1] = {s->batch};
    if (!pointer(a[5], "first", at::kInt, batch, device, true, &first) || !pointer(a[6], "count", at::kInt, batch, device, true, &count) ||
        !current_stream(device, &stream))
        return nullptr;
    if (k->size(1) > INT32_MAX) return PyLong_FromLong(GKV_ERR_UNSUPPORTED);
    const int32_t tokens = (int32_t)k->size(1);
    const gkv_status st = read ? g_read(s, k->data_ptr(), v->data_ptr(), strides[0], strides[1], strides[2], (const int32_t*)first,
                                        (const int32_t*)count, tokens, stream)
                               : g_write(s, k->data_ptr(), v->data_ptr(), strides[0], strides[1], strides[2], (const int32_t*)first,
                                         (const int32_t*)count, tokens, stream);
    return PyLong_FromLong(st);
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// attn(store, device, length, max_len, q, k_new, v_new, prefix, out, lse, workspace, workspace_bytes) -> status
PyObject* attn(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    if (!arguments(n, 12, "attn")) return nullptr;
    const gkv_store* s = address<const gkv_store>(a[0]);
    const int device = (int)PyLong_AsLong(a[1]);
    const long max_len = PyLong_AsLong(a[3]);
    const gkv_prefix* prefix = address<const gkv_prefix>(a[7]);
    void* ws = address<void>(a[10]);
    const uint64_t ws_bytes = PyLong_AsUnsignedLongLong(a[11]);
    if (PyErr_Occurred()) return nullptr;
    if (max_len < INT32_MIN || max_len > INT32_MAX) return PyLong_FromLong(GKV_ERR_INVALID_ARG);
    const int64_t batch[1] = {s->batch}, qs[3] = {s->batch, s->n_q_heads, s->head_dim}, kvs[3] = {s->batch, s->n_kv_heads, s->head_dim},
                  ls[2] = {s->batch, s->n_q_heads};
    void *length, *q, *k_new, *v_new, *out, *lse, *stream;
    if (!pointer(a[2], "length", at::kInt, batch, device, false, &length) || !pointer(a[4], "q", at::kBFloat16, qs, device, false, &q) ||
        !pointer(a[5], "k_new", at::kBFloat16, kvs, device, true, &k_new) || !pointer(a[6], "v_new", at::kBFloat16, kvs, device, true, &v_new) ||
        !pointer(a[8], "out", at::kBFloat16, qs, device, false, &out) || !pointer(a[9], "lse", at::kFloat, ls, device, true, &lse) ||
        !current_stream(device, &stream))
        return nullptr;
    return PyLong_FromLong(g_attn(s, (const int32_t*)length, (int32_t)max_len, q, k_new, v_new, prefix, out, (float*)lse, ws, ws_bytes, stream));
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// in_use((stream, device, tensor, ...)): the tensors, allocated on that stream (its cudaStream_t), have been given to work on the
// current stream. If that is another one, the allocator is told, so that it does not hand their memory out again before that work is done.
PyObject* in_use(PyObject*, PyObject* held) try {
    if (!PyTuple_Check(held) || PyTuple_GET_SIZE(held) < 2) {
        PyErr_SetString(PyExc_TypeError, "in_use takes a tuple (stream, device, tensor, ...)");
        return nullptr;
    }
    const void* home = address<const void>(PyTuple_GET_ITEM(held, 0));
    const int device = (int)PyLong_AsLong(PyTuple_GET_ITEM(held, 1));
    if (PyErr_Occurred()) return nullptr;
    const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(device);
    if (current.stream() != home)
        for (Py_ssize_t i = 2; i < PyTuple_GET_SIZE(held); ++i) {
            const at::Tensor* t = tensor(PyTuple_GET_ITEM(held, i), "in_use");
            if (!t) return nullptr;
            c10::cuda::CUDACachingAllocator::recordStream(t->storage().data_ptr(), current);
        }
    Py_RETURN_NONE;
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

PyMethodDef g_methods[] = {{"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
                           {"copy", (PyCFunction)(void (*)(void))copy, METH_FASTCALL, nullptr},
                           {"attn", (PyCFunction)(void (*)(void))attn, METH_FASTCALL, nullptr},
                           {"in_use", (PyCFunction)in_use, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_gkv_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#ifndef GKV_BUILT_FOR
#define GKV_BUILT_FOR "unknown"
#endif

PyMODINIT_FUNC PyInit__gkv_torch(void) {
    PyObject* m = PyModule_Create(&g_module);
    if (m && PyModule_AddStringConstant(m, "built_for", GKV_BUILT_FOR) != 0) Py_CLEAR(m);
    return m;
}
