// Python side of the KV-cache calls: checks of the tensors, marshalling, allocation of the results.
//
// A decode round is a few microseconds of device time for each of these calls, so what the interpreter adds counts: as
// Python with ctypes the checks, the argument conversion and the allocations took 8 us for an append and 17 us for an
// attention call, more than the kernels.  The C entry points are handed over by address (init), so that this module
// serves whichever build of the library is loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "hos.h"

namespace {

decltype(&hos_kv_append) p_append;
decltype(&hos_kv_read) p_read;
decltype(&hos_paged_attention) p_attention;
decltype(&hos_paged_attention_workspace_bytes) p_workspace;

constexpr int STATUS_TOO_SHORT = 1;              // not an error of the library: the caller lengthens its status words and calls again

struct Cache {
    hos_kv_cache c;
    at::ScalarType type;
    c10::DeviceIndex device;
    at::Tensor status;
    cudaStream_t home;                           // that the status words were allocated on
    int32_t* words(c10::cuda::CUDAStream st) const {
        // their memory is not given to anyone else before a call on another stream is done with it
        if (st.stream() != home) c10::cuda::CUDACachingAllocator::recordStream(status.storage().data_ptr(), st);
        return status.mutable_data_ptr<int32_t>();
    }
};
void drop(PyObject* capsule) { delete static_cast<Cache*>(PyCapsule_GetPointer(capsule, "hos.kv_cache")); }
Cache* cache_of(PyObject* o) { return static_cast<Cache*>(PyCapsule_GetPointer(o, "hos.kv_cache")); }

const at::Tensor* tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: expected a tensor", what);
        return nullptr;
    }
    return &THPVariable_Unpack(o);
}

// The batch's three tensors.
bool batch_of(const Cache* c, PyObject* off_o, PyObject* len_o, PyObject* table_o, int64_t n_tokens, int64_t max_new, hos_kv_batch* b) {
    const at::Tensor* off = tensor(off_o, "tok_off");
    const at::Tensor* len = off ? tensor(len_o, "kv_len") : nullptr;
    const at::Tensor* table = len ? tensor(table_o, "page_table") : nullptr;
    if (!table) return false;
    for (const at::Tensor* t : {off, len, table})
        if (t->scalar_type() != at::kInt || !t->is_cuda() || t->get_device() != c->device) {
            PyErr_SetString(PyExc_TypeError, "tok_off, kv_len, page_table: expected int32 tensors on the cache's device");
            return false;
        }
    if (off->dim() != 1 || len->dim() != 1 || table->dim() != 2) {
        PyErr_SetString(PyExc_ValueError, "tok_off and kv_len must have one dimension, page_table two");
        return false;
    }
    const int64_t n_seq = len->size(0), width = table->size(1);
    if (off->size(0) != n_seq + 1 || table->size(0) != n_seq) {
        PyErr_SetString(PyExc_ValueError, "tok_off must have n_seq + 1 entries, kv_len n_seq, page_table n_seq rows");
        return false;
    }
    if ((width > 1 && table->stride(1) != 1) || !off->is_contiguous() || !len->is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "tok_off, kv_len and the rows of page_table must be dense");
        return false;
    }
    if (n_seq > INT32_MAX || width > INT32_MAX || n_tokens > INT32_MAX || max_new > INT32_MAX || max_new < INT32_MIN) {
        PyErr_SetString(PyExc_ValueError, "sizes beyond 32 bits");
        return false;
    }
    *b = hos_kv_batch{(int32_t)n_seq, (int32_t)n_tokens, (int32_t)max_new, (int32_t)width, off->const_data_ptr<int32_t>(),
                      len->const_data_ptr<int32_t>(), table->const_data_ptr<int32_t>(), n_seq > 1 ? table->stride(0) : width};
    return true;
}

// A [tokens][heads][head_dim] tensor of the cache's type.
const at::Tensor* rows(const Cache* c, PyObject* o, const char* what) {
    const at::Tensor* t = tensor(o, what);
    if (!t) return nullptr;
    if (t->scalar_type() != c->type || !t->is_cuda() || t->get_device() != c->device) {
        PyErr_Format(PyExc_TypeError, "%s: expected a tensor of the cache's dtype on its device", what);
        return nullptr;
    }
    if (t->dim() != 3 || t->size(2) != c->c.head_dim) {
        PyErr_Format(PyExc_ValueError, "%s: expected [tokens][heads][%d]", what, (int)c->c.head_dim);
        return nullptr;
    }
    if (t->stride(2) != 1) {
        PyErr_Format(PyExc_ValueError, "%s: the elements of a head must be dense", what);
        return nullptr;
    }
    if (t->requires_grad() && c10::GradMode::is_enabled()) {     // the results would carry no graph
        PyErr_Format(PyExc_ValueError, "%s requires grad, and there is no backward pass: detach it, or call under torch.no_grad()", what);
        return nullptr;
    }
    return t;
}

// Strides of a [tokens][heads][head_dim] tensor.  Those of a single token or head mean nothing (and torch leaves anything there).
int64_t token_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1) * t.size(2); }
int64_t head_stride(const at::Tensor& t) { return t.size(1) > 1 ? t.stride(1) : t.size(2); }

bool arity(Py_ssize_t have, Py_ssize_t want) {
    if (have == want) return true;
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return false;
}

// torch's own errors (out of memory, for one) become Python exceptions.
template <typename F> PyObject* guarded(F&& f) {
    try {
        return f();
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// init(append, read, attention, workspace_bytes): addresses of the C entry points
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 4)) return nullptr;
    void* p[4];
    for (int i = 0; i < 4; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    p_append = reinterpret_cast<decltype(p_append)>(p[0]);
    p_read = reinterpret_cast<decltype(p_read)>(p[1]);
    p_attention = reinterpret_cast<decltype(p_attention)>(p[2]);
    p_workspace = reinterpret_cast<decltype(p_workspace)>(p[3]);
    Py_RETURN_NONE;
}

// cache(address of a hos_kv_cache, device index): handle
PyObject* cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 2)) return nullptr;
    const void* src = PyLong_AsVoidPtr(a[0]);
    const long device = PyLong_AsLong(a[1]);
    if (PyErr_Occurred()) return nullptr;
    Cache* c = new Cache{*static_cast<const hos_kv_cache*>(src), at::kHalf, (c10::DeviceIndex)device, at::Tensor(), nullptr};
    if (c->c.type == HOS_TYPE_BF16) c->type = at::kBFloat16;
    return PyCapsule_New(c, "hos.kv_cache", drop);
}

// set_status(handle, words): int32, allocated on the current stream
PyObject* set_status(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (!arity(n, 2)) return nullptr;
        Cache* c = cache_of(a[0]);
        const at::Tensor* t = c ? tensor(a[1], "status") : nullptr;
        if (!t) return nullptr;
        c->status = *t;
        c->home = c10::cuda::getCurrentCUDAStream(c->device).stream();
        Py_RETURN_NONE;
    });
}

// append(handle, k, v, tok_off, kv_len, page_table): error code
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (!arity(n, 6)) return nullptr;
        const Cache* c = cache_of(a[0]);
        const at::Tensor* k = c ? rows(c, a[1], "k") : nullptr;
        const at::Tensor* v = k ? rows(c, a[2], "v") : nullptr;
        if (!v) return nullptr;
        if (k->size(1) != c->c.n_kv_heads || v->size(1) != c->c.n_kv_heads || k->size(0) != v->size(0)) {
            PyErr_SetString(PyExc_ValueError, "k and v must be [n_tokens][n_kv_heads][head_dim]");
            return nullptr;
        }
        hos_kv_batch b;
        if (!batch_of(c, a[3], a[4], a[5], k->size(0), k->size(0), &b)) return nullptr;
        if (b.n_seq > c->status.numel()) return PyLong_FromLong(STATUS_TOO_SHORT);
        const c10::cuda::CUDAGuard guard(c->device);
        const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream(c->device);
        return PyLong_FromLong(p_append(&c->c, &b, k->const_data_ptr(), v->const_data_ptr(), token_stride(*k), head_stride(*k),
                                        token_stride(*v), head_stride(*v), c->words(st), st.stream()));
    });
}

// read(handle, tok_off, kv_len, page_table, n_tokens, k or None, v or None): (error code, k, v)
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (!arity(n, 7)) return nullptr;
        const Cache* c = cache_of(a[0]);
        if (!c) return nullptr;
        const long long n_tok = PyLong_AsLongLong(a[4]);
        if (PyErr_Occurred()) return nullptr;
        if (n_tok < 0) {
            PyErr_SetString(PyExc_ValueError, "n_tokens must not be negative");
            return nullptr;
        }
        hos_kv_batch b;
        if (!batch_of(c, a[1], a[2], a[3], n_tok, n_tok, &b)) return nullptr;
        if (b.n_seq > c->status.numel()) return Py_BuildValue("iOO", STATUS_TOO_SHORT, Py_None, Py_None);
        const c10::cuda::CUDAGuard guard(c->device);
        at::Tensor out[2];
        for (int i = 0; i < 2; ++i) {
            if (a[5 + i] == Py_None) {
                out[i] = at::empty({n_tok, c->c.n_kv_heads, c->c.head_dim}, at::TensorOptions().dtype(c->type).device(at::kCUDA, c->device));
                continue;
            }
            const at::Tensor* t = rows(c, a[5 + i], "out");
            if (!t) return nullptr;
            if (t->size(0) != n_tok || t->size(1) != c->c.n_kv_heads || !t->is_contiguous()) {
                PyErr_SetString(PyExc_ValueError, "out tensors must be dense [n_tokens][n_kv_heads][head_dim]");
                return nullptr;
            }
            out[i] = *t;
        }
        const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream(c->device);
        const int rc = p_read(&c->c, &b, out[0].mutable_data_ptr(), out[1].mutable_data_ptr(), c->words(st), st.stream());
        return Py_BuildValue("iNN", rc, THPVariable_Wrap(out[0]), THPVariable_Wrap(out[1]));
    });
}

// attention(handle, q, tok_off, kv_len, page_table, max_new, sm_scale or None, causal, window, want_lse, out or None, ws or None):
// (error code, out, lse or None)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (!arity(n, 12)) return nullptr;
        const Cache* c = cache_of(a[0]);
        const at::Tensor* q = c ? rows(c, a[1], "q") : nullptr;
        if (!q) return nullptr;
        const long long max_new = PyLong_AsLongLong(a[5]), window = PyLong_AsLongLong(a[8]);
        const double scale = a[6] == Py_None ? 1.0 / std::sqrt((double)c->c.head_dim) : PyFloat_AsDouble(a[6]);
        const int causal = PyObject_IsTrue(a[7]), want_lse = PyObject_IsTrue(a[9]);
        if (PyErr_Occurred()) return nullptr;
        if (window > INT32_MAX || window < INT32_MIN || q->size(1) > INT32_MAX) {
            PyErr_SetString(PyExc_ValueError, "sizes beyond 32 bits");
            return nullptr;
        }
        hos_kv_batch b;
        if (!batch_of(c, a[2], a[3], a[4], q->size(0), max_new, &b)) return nullptr;
        if (b.n_seq > c->status.numel()) return Py_BuildValue("iOO", STATUS_TOO_SHORT, Py_None, Py_None);
        const c10::cuda::CUDAGuard guard(c->device);
        at::Tensor out, lse, ws;
        if (a[10] == Py_None) {
            out = at::empty(q->sizes(), at::TensorOptions().dtype(c->type).device(at::kCUDA, c->device));
        } else {
            const at::Tensor* t = rows(c, a[10], "out");
            if (!t) return nullptr;
            if (t->sizes() != q->sizes()) {
                PyErr_SetString(PyExc_ValueError, "out must have the shape of q");
                return nullptr;
            }
            if ((t->size(0) > 1 && t->stride(0) == 0) || (t->size(1) > 1 && t->stride(1) == 0)) {
                PyErr_SetString(PyExc_ValueError, "out: several rows in one place (an expanded tensor)");
                return nullptr;
            }
            out = *t;
        }
        const int heads = (int)q->size(1);
        if (want_lse) lse = at::empty({q->size(0), heads}, at::TensorOptions().dtype(at::kFloat).device(at::kCUDA, c->device));
        const int64_t need = (int64_t)p_workspace(&c->c, &b, heads);
        if (a[11] != Py_None) {
            const at::Tensor* t = tensor(a[11], "ws");
            if (!t) return nullptr;
            if (t->scalar_type() != at::kByte || !t->is_cuda() || t->get_device() != c->device || !t->is_contiguous()) {
                PyErr_SetString(PyExc_TypeError, "ws: expected a dense uint8 tensor on the cache's device");
                return nullptr;
            }
            ws = *t;
        } else {
            ws = at::empty({need}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, c->device));
        }
        const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream(c->device);
        const int rc = p_attention(&c->c, &b, q->const_data_ptr(), token_stride(*q), head_stride(*q), heads, (float)scale, causal, (int)window,
                                   out.mutable_data_ptr(), token_stride(out), head_stride(out), want_lse ? lse.mutable_data_ptr<float>() : nullptr,
                                   c->words(st), ws.mutable_data_ptr(), (size_t)ws.numel(), st.stream());
        return Py_BuildValue("iNN", rc, THPVariable_Wrap(out), want_lse ? THPVariable_Wrap(lse) : Py_NewRef(Py_None));
    });
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"init", FAST(init)}, {"cache", FAST(cache)}, {"set_status", FAST(set_status)}, {"append", FAST(append)},
                         {"read", FAST(read)}, {"attention", FAST(attention)}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv() { return PyModule_Create(&module); }
