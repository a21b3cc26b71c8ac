// Python module that hands torch tensors to the key/value store, paged cache and rotary calls of the C ABI: it checks types, shapes, devices and
// strides and makes the call, all in one step. (Through ctypes the same checks and conversions took 7 to 8 us a call, more than
// most decode-sized kernels run; here they take well under one.) It holds no state but the addresses of the library's functions,
// so that it serves every build of the library.
#include <Python.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <sstream>
#include <string>

#include "gkv.h"

namespace {

decltype(&gkv_store_write) g_write;
decltype(&gkv_store_read) g_read;
decltype(&gkv_store_attn) g_attn;
decltype(&gkv_pages_append) g_pages_append;
decltype(&gkv_pages_read) g_pages_read;
decltype(&gkv_pages_attn) g_pages_attn;
decltype(&gkv_rotary_apply) g_rotary;

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
// A tensor that a call has written counts as changed, so that a backward pass that has kept it says so instead of using what it holds now.
void changed(PyObject* o) {
    if (o == Py_None) return;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// The calls record nothing for a backward pass. What needs a gradient is refused where one is being recorded, as torch refuses it of its
// own functions that write to given tensors.
bool outside_autograd(PyObject* o, const char* what) {
    if (o == Py_None || !c10::GradMode::is_enabled() || !THPVariable_Unpack(o).requires_grad()) return true;
    PyErr_Format(PyExc_ValueError, "%s requires grad, and this call records nothing for a backward pass: make it under torch.no_grad() (in "
                 "a torch.autograd.Function, say), and turn the gradients with transpose=True", what);
    return false;
}
bool arguments(Py_ssize_t n, Py_ssize_t want, const char* what) {
    if (n != want) PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", what, want, n);
    return n == want;
}
template <typename T>
T* address(PyObject* o) { return reinterpret_cast<T*>(PyLong_AsUnsignedLongLong(o)); }

// bind(write, read, attn, pages append, pages read, pages attn, rotary): addresses of the library's functions
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arguments(n, 7, "bind")) return nullptr;
    g_write = reinterpret_cast<decltype(g_write)>(PyLong_AsUnsignedLongLong(a[0]));
    g_read = reinterpret_cast<decltype(g_read)>(PyLong_AsUnsignedLongLong(a[1]));
    g_attn = reinterpret_cast<decltype(g_attn)>(PyLong_AsUnsignedLongLong(a[2]));
    g_pages_append = reinterpret_cast<decltype(g_pages_append)>(PyLong_AsUnsignedLongLong(a[3]));
    g_pages_read = reinterpret_cast<decltype(g_pages_read)>(PyLong_AsUnsignedLongLong(a[4]));
    g_pages_attn = reinterpret_cast<decltype(g_pages_attn)>(PyLong_AsUnsignedLongLong(a[5]));
    g_rotary = reinterpret_cast<decltype(g_rotary)>(PyLong_AsUnsignedLongLong(a[6]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

// k and v, bf16 [batch][tokens][heads][head_dim] with the same strides (0 for steps that are not taken), the last of them 1.
bool tokens_of(PyObject* ok, PyObject* ov, int64_t batch, int64_t heads, int64_t head_dim, int device, const at::Tensor** pk, const at::Tensor** pv,
               int64_t (&strides)[3]) {
    const at::Tensor *k = tensor(ok, "k"), *v = k ? tensor(ov, "v") : nullptr;
    if (!v) return false;
    for (const at::Tensor* t : {k, v}) {
        if (t->scalar_type() != at::kBFloat16 || t->dim() != 4 || t->size(0) != batch || t->size(2) != heads || t->size(3) != head_dim ||
            t->sizes() != k->sizes() || !t->is_cuda() || t->get_device() != device) {
            std::ostringstream m;
            m << (t == k ? "k" : "v") << ": a BFloat16 tensor [" << batch << "][tokens][" << heads << "][" << head_dim << "] on cuda:" << device
              << " is needed, got " << type_name(t->scalar_type()) << " " << t->sizes() << " on " << t->device();
            PyErr_SetString(PyExc_ValueError, m.str().c_str());
            return false;
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
            return false;
        }
    }
    *pk = k;
    *pv = v;
    return true;
}

// copy(read, store, device, k, v, first, count) -> status
PyObject* copy(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    if (!arguments(n, 7, "copy")) return nullptr;
    const bool read = a[0] == Py_True;
    const gkv_store* s = address<const gkv_store>(a[1]);
    const int device = (int)PyLong_AsLong(a[2]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *k, *v;
    int64_t strides[3];
    if (!tokens_of(a[3], a[4], s->batch, s->n_kv_heads, s->head_dim, device, &k, &v, strides)) return nullptr;
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
    if (read && st == GKV_OK) {
        changed(a[3]);
        changed(a[4]);
    }
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
    const gkv_status st = g_attn(s, (const int32_t*)length, (int32_t)max_len, q, k_new, v_new, prefix, out, (float*)lse, ws, ws_bytes, stream);
    if (st == GKV_OK) {
        changed(a[8]);
        changed(a[9]);
    }
    return PyLong_FromLong(st);
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// An int32 tensor [n0][n1] on the device, any strides; None gives NULL where that is allowed.
bool int_table(PyObject* o, const char* what, int64_t n0, int64_t n1, int device, bool optional, const int32_t** out, int64_t (&strides)[2]) {
    *out = nullptr;
    strides[0] = strides[1] = 0;
    if (optional && o == Py_None) return true;
    const at::Tensor* t = tensor(o, what);
    if (!t) return false;
    if (t->scalar_type() != at::kInt || t->dim() != 2 || (n0 >= 0 && t->size(0) != n0) || (n1 >= 0 && t->size(1) != n1) || !t->is_cuda() ||
        t->get_device() != device) {
        std::ostringstream m;
        m << what << ": an Int tensor [" << (n0 < 0 ? "batch" : std::to_string(n0)) << "][" << (n1 < 0 ? "places" : std::to_string(n1))
          << "] on cuda:" << device << " is needed, got " << type_name(t->scalar_type()) << " " << t->sizes() << " on " << t->device();
        PyErr_SetString(PyExc_ValueError, m.str().c_str());
        return false;
    }
    for (int i = 0; i < 2; ++i) strides[i] = t->size(i) == 1 ? 0 : t->stride(i);
    *out = (const int32_t*)t->data_ptr();
    return true;
}
// The table of a paged call: [batch][places], the places of a sequence next to one another.
bool page_table(PyObject* o, int device, gkv_page_table* out) {
    int64_t st[2];
    if (!int_table(o, "table", -1, -1, device, false, &out->page, st)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX || (t.size(1) > 1 && st[1] != 1)) {
        PyErr_SetString(PyExc_ValueError, "table: the places of a sequence have to lie next to one another, and both sizes to fit 32 bits");
        return false;
    }
    out->stride = st[0];
    out->batch = (int32_t)t.size(0);
    out->width = (int32_t)t.size(1);
    return true;
}
// bf16 rows [batch][heads][head_dim] whose heads lie next to one another; *stride: from a sequence to the next. None gives NULL where
// that is allowed.
bool heads_of(PyObject* o, const char* what, int64_t batch, int64_t heads, int64_t head_dim, int device, bool optional, void** out, int64_t* stride) {
    *out = nullptr;
    *stride = 0;
    if (optional && o == Py_None) return true;
    const at::Tensor* t = tensor(o, what);
    if (!t) return false;
    const int64_t shape[3] = {batch, heads, head_dim};
    if (t->scalar_type() != at::kBFloat16 || t->sizes() != at::IntArrayRef(shape) || !t->is_cuda() || t->get_device() != device ||
        t->stride(2) != 1 || (heads > 1 && t->stride(1) != head_dim)) {
        std::ostringstream m;
        m << what << ": a BFloat16 tensor " << at::IntArrayRef(shape) << " on cuda:" << device << " whose heads lie next to one another is needed, got "
          << type_name(t->scalar_type()) << " " << t->sizes() << " with strides " << t->strides() << " on " << t->device();
        PyErr_SetString(PyExc_ValueError, m.str().c_str());
        return false;
    }
    *out = t->data_ptr();
    *stride = batch > 1 ? t->stride(0) : 0;
    return true;
}

// pages_copy(read, pages, device, table, k, v, first, count, rotary, pos) -> status
PyObject* pages_copy(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    if (!arguments(n, 10, "pages_copy")) return nullptr;
    const bool read = a[0] == Py_True;
    const gkv_pages* s = address<const gkv_pages>(a[1]);
    const int device = (int)PyLong_AsLong(a[2]);
    const gkv_rotary* rotary = address<const gkv_rotary>(a[8]);
    if (PyErr_Occurred()) return nullptr;
    gkv_page_table table;
    if (!page_table(a[3], device, &table)) return nullptr;
    const at::Tensor *k, *v;
    int64_t strides[3], ps[2];
    if (!tokens_of(a[4], a[5], table.batch, s->n_kv_heads, s->head_dim, device, &k, &v, strides)) return nullptr;
    void *first, *count, *stream;
    const int32_t* pos;
    const int64_t batch[1] = {table.batch};
    if (!pointer(a[6], "first", at::kInt, batch, device, true, &first) || !pointer(a[7], "count", at::kInt, batch, device, true, &count) ||
        !int_table(a[9], "pos", table.batch, k->size(1), device, true, &pos, ps) || !current_stream(device, &stream))
        return nullptr;
    if (k->size(1) > INT32_MAX) return PyLong_FromLong(GKV_ERR_UNSUPPORTED);
    const int32_t tokens = (int32_t)k->size(1);
    const gkv_status st =
        read ? g_pages_read(s, &table, k->data_ptr(), v->data_ptr(), strides[0], strides[1], strides[2], (const int32_t*)first, (const int32_t*)count,
                            tokens, stream)
             : g_pages_append(s, &table, k->data_ptr(), v->data_ptr(), strides[0], strides[1], strides[2], (const int32_t*)first,
                              (const int32_t*)count, tokens, rotary, pos, ps[0], ps[1], stream);
    if (read && st == GKV_OK) {
        changed(a[4]);
        changed(a[5]);
    }
    return PyLong_FromLong(st);
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// pages_attn(pages, device, max_batch, table, length, max_len, q, k_new, v_new, rotary, pos, out, lse, workspace, workspace_bytes) -> status
PyObject* pages_attn(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    if (!arguments(n, 15, "pages_attn")) return nullptr;
    const gkv_pages* s = address<const gkv_pages>(a[0]);
    const int device = (int)PyLong_AsLong(a[1]);
    const long max_batch = PyLong_AsLong(a[2]), max_len = PyLong_AsLong(a[5]);
    const gkv_rotary* rotary = address<const gkv_rotary>(a[9]);
    void* ws = address<void>(a[13]);
    const uint64_t ws_bytes = PyLong_AsUnsignedLongLong(a[14]);
    if (PyErr_Occurred()) return nullptr;
    if (max_len < INT32_MIN || max_len > INT32_MAX) return PyLong_FromLong(GKV_ERR_INVALID_ARG);
    gkv_page_table table;
    if (!page_table(a[3], device, &table)) return nullptr;
    if (table.batch > max_batch) {
        PyErr_Format(PyExc_ValueError, "the table has %d sequences, the workspace is for %ld", (int)table.batch, max_batch);
        return nullptr;
    }
    const int64_t b = table.batch, batch[1] = {b}, qs[3] = {b, s->n_q_heads, s->head_dim}, ls[2] = {b, s->n_q_heads};
    void *length, *q, *k_new, *v_new, *pos, *out, *lse, *stream;
    int64_t q_stride, k_stride, v_stride;
    if (!pointer(a[4], "length", at::kInt, batch, device, false, &length) ||
        !heads_of(a[6], "q", b, s->n_q_heads, s->head_dim, device, false, &q, &q_stride) ||
        !heads_of(a[7], "k_new", b, s->n_kv_heads, s->head_dim, device, true, &k_new, &k_stride) ||
        !heads_of(a[8], "v_new", b, s->n_kv_heads, s->head_dim, device, true, &v_new, &v_stride) ||
        !pointer(a[10], "pos", at::kInt, batch, device, true, &pos) || !pointer(a[11], "out", at::kBFloat16, qs, device, false, &out) ||
        !pointer(a[12], "lse", at::kFloat, ls, device, true, &lse) || !current_stream(device, &stream))
        return nullptr;
    if (k_new && v_new && k_stride != v_stride) {
        PyErr_Format(PyExc_ValueError, "k_new, v_new: sequences are %lld and %lld elements apart: the two have to agree", (long long)k_stride,
                     (long long)v_stride);
        return nullptr;
    }
    const gkv_status st = g_pages_attn(s, &table, (const int32_t*)length, (int32_t)max_len, q, q_stride, k_new, v_new, k_stride, rotary,
                                       (const int32_t*)pos, out, (float*)lse, ws, ws_bytes, stream);
    if (st == GKV_OK) {
        changed(a[11]);
        changed(a[12]);
    }
    return PyLong_FromLong(st);
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// Rows [batch][tokens][heads][head_dim] of a rotation; strides of steps that are not taken are 0.
bool rotary_rows(PyObject* ox, PyObject* oy, const char* what, const at::Tensor* like, int64_t head_dim, int device, gkv_rotary_rows* r) {
    const at::Tensor* x = tensor(ox, what);
    const at::Tensor* y = !x || oy == Py_None ? x : tensor(oy, what);
    if (!y) return false;
    if (!like) like = x;
    const at::ScalarType type = like->scalar_type();
    for (const at::Tensor* t : {x, y})
        if ((type != at::kBFloat16 && type != at::kHalf && type != at::kFloat) || t->scalar_type() != type || t->dim() != 4 ||
            t->sizes() != x->sizes() || t->size(0) != like->size(0) || t->size(1) != like->size(1) || t->size(3) != head_dim ||
            t->stride(3) != 1 || !t->is_cuda() || t->get_device() != device || t->size(2) > INT32_MAX) {
            std::ostringstream m;
            m << what << (t == x ? "" : "_out") << ": a BFloat16, Half or Float tensor [batch][tokens][heads][" << head_dim << "] on cuda:" << device
              << " with a last stride of 1 (all of them of one type, batch and number of tokens) is needed, got " << type_name(t->scalar_type())
              << " " << t->sizes() << " with strides " << t->strides() << " on " << t->device();
            PyErr_SetString(PyExc_ValueError, m.str().c_str());
            return false;
        }
    r->x = x->data_ptr();
    r->y = y->data_ptr();
    for (int i = 0; i < 3; ++i) {
        r->x_stride[i] = x->size(i) == 1 ? 0 : x->stride(i);
        r->y_stride[i] = y->size(i) == 1 ? 0 : y->stride(i);
    }
    r->n_heads = (int32_t)x->size(2);
    return true;
}

// rotary(rotary, device, pos, q, k, q_out, k_out, count, transpose) -> status
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    if (!arguments(n, 9, "rotary")) return nullptr;
    const gkv_rotary* r = address<const gkv_rotary>(a[0]);
    const int device = (int)PyLong_AsLong(a[1]);
    const int transpose = PyObject_IsTrue(a[8]);
    if (PyErr_Occurred()) return nullptr;
    gkv_rotary_rows q, k;
    const bool two = a[4] != Py_None;
    if (!rotary_rows(a[3], a[5], "q", nullptr, r->head_dim, device, &q)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(a[3]);
    if (two && !rotary_rows(a[4], a[6], "k", &t, r->head_dim, device, &k)) return nullptr;
    if (!two && a[6] != Py_None) {
        PyErr_SetString(PyExc_ValueError, "k_out without k");
        return nullptr;
    }
    if (!outside_autograd(a[3], "q") || !outside_autograd(a[4], "k") || !outside_autograd(a[5], "q_out") || !outside_autograd(a[6], "k_out"))
        return nullptr;
    const int32_t* pos;
    int64_t ps[2];
    void *count, *stream;
    const int64_t batch[1] = {t.size(0)};
    if (!int_table(a[2], "pos", t.size(0), t.size(1), device, false, &pos, ps) || !pointer(a[7], "count", at::kInt, batch, device, true, &count) ||
        !current_stream(device, &stream))
        return nullptr;
    if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) return PyLong_FromLong(GKV_ERR_UNSUPPORTED);
    const int type = t.scalar_type() == at::kFloat ? GKV_TYPE_FP32 : t.scalar_type() == at::kHalf ? GKV_TYPE_FP16 : GKV_TYPE_BF16;
    const gkv_status st = g_rotary(r, type, (int32_t)t.size(0), (int32_t)t.size(1), pos, ps[0], ps[1], (const int32_t*)count, &q, two ? &k : nullptr,
                                   transpose, stream);
    if (st == GKV_OK) {
        changed(a[5] != Py_None ? a[5] : a[3]);
        if (two) changed(a[6] != Py_None ? a[6] : a[4]);
    }
    return PyLong_FromLong(st);
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
                           {"pages_copy", (PyCFunction)(void (*)(void))pages_copy, METH_FASTCALL, nullptr},
                           {"pages_attn", (PyCFunction)(void (*)(void))pages_attn, METH_FASTCALL, nullptr},
                           {"rotary", (PyCFunction)(void (*)(void))rotary, METH_FASTCALL, nullptr},
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
