// Python side of the KV-cache calls: checks of the tensors, marshalling, allocation of the results.
//
// A decode round is a few microseconds of device time for each of these calls, so what the interpreter adds counts: as
// Python with ctypes the checks, the argument conversion and the allocations took 8 us for an append and 17 us for an
// attention call, more than the kernels.  The C entry points are handed over by address (init), so that this module
// serves whichever build of the library is loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <vector>

#include "hos.h"

namespace {

decltype(&hos_kv_append) p_append;
decltype(&hos_kv_read) p_read;
decltype(&hos_paged_attention) p_attention;
decltype(&hos_paged_attention_workspace_bytes) p_workspace;
decltype(&hos_kv_resize) p_resize;
decltype(&hos_kv_resize_workspace_bytes) p_resize_workspace;
decltype(&hos_kv_fork) p_fork;
decltype(&hos_kv_compact) p_compact;
decltype(&hos_kv_compact_workspace_bytes) p_compact_workspace;
decltype(&hos_kv_copy_pages) p_copy_pages;
decltype(&hos_verify_drafts) p_verify;

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

// init(addresses of the C entry points, in the order below)
template <typename P> void set(P& entry, PyObject* address) { entry = reinterpret_cast<P>(PyLong_AsVoidPtr(address)); }
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 11)) return nullptr;
    set(p_append, a[0]);
    set(p_read, a[1]);
    set(p_attention, a[2]);
    set(p_workspace, a[3]);
    set(p_resize, a[4]);
    set(p_resize_workspace, a[5]);
    set(p_fork, a[6]);
    set(p_compact, a[7]);
    set(p_compact_workspace, a[8]);
    set(p_copy_pages, a[9]);
    set(p_verify, a[10]);
    if (PyErr_Occurred()) return nullptr;
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

// ---- the pages of a cache ------------------------------------------------------------------------------------------

// A dense int32 (or float32) tensor of one dimension on `device` (-1: any CUDA device) with `size` elements (-1: any).
const at::Tensor* vector(PyObject* o, const char* what, at::ScalarType type, int device, int64_t size) {
    const at::Tensor* t = tensor(o, what);
    if (!t) return nullptr;
    if (t->scalar_type() != type || !t->is_cuda() || (device >= 0 && t->get_device() != device)) {
        PyErr_Format(PyExc_TypeError, "%s: expected a CUDA tensor of %s%s", what, type == at::kInt ? "int32" : "float32",
                     device >= 0 ? " on the same device as the others" : "");
        return nullptr;
    }
    if (t->dim() != 1 || !t->is_contiguous() || (size >= 0 && t->size(0) != size)) {
        if (size >= 0) PyErr_Format(PyExc_ValueError, "%s: expected one dense dimension of %lld", what, (long long)size);
        else PyErr_Format(PyExc_ValueError, "%s: expected one dense dimension", what);
        return nullptr;
    }
    if (t->size(0) > INT32_MAX) {
        PyErr_SetString(PyExc_ValueError, "sizes beyond 32 bits");
        return nullptr;
    }
    return t;
}

// refs, page_table and kv_len; device -1 and n_seq -1: whatever the first of them has.
bool state_of(PyObject* refs_o, PyObject* table_o, PyObject* len_o, long long page_size, int device, int64_t n_pages, int64_t n_seq, int64_t width,
              hos_kv_pages* p) {
    const at::Tensor* refs = vector(refs_o, "refs", at::kInt, device, n_pages);
    if (!refs) return false;
    const at::Tensor* len = vector(len_o, "kv_len", at::kInt, refs->get_device(), n_seq);
    const at::Tensor* table = len ? tensor(table_o, "page_table") : nullptr;
    if (!table) return false;
    if (table->scalar_type() != at::kInt || !table->is_cuda() || table->get_device() != refs->get_device()) {
        PyErr_SetString(PyExc_TypeError, "page_table: expected a CUDA tensor of int32 on the same device as the others");
        return false;
    }
    if (table->dim() != 2 || table->size(0) != len->size(0) || (width >= 0 && table->size(1) != width) || (table->size(1) > 1 && table->stride(1) != 1)) {
        PyErr_SetString(PyExc_ValueError, "page_table: expected [n_seq][pages] with dense rows");
        return false;
    }
    if (table->size(0) > 1 && table->stride(0) < table->size(1)) {
        PyErr_SetString(PyExc_ValueError, "page_table: rows must not overlap");
        return false;
    }
    if (table->size(1) > INT32_MAX || page_size > INT32_MAX || page_size < 1) {
        PyErr_SetString(PyExc_ValueError, "sizes beyond 32 bits, or no page size");
        return false;
    }
    *p = hos_kv_pages{(int32_t)refs->size(0), (int32_t)page_size, (int32_t)len->size(0), (int32_t)table->size(1), refs->mutable_data_ptr<int32_t>(),
                      len->mutable_data_ptr<int32_t>(), table->mutable_data_ptr<int32_t>(), table->size(0) > 1 ? table->stride(0) : table->size(1)};
    return true;
}

// The int32 results of a call and its workspace, cut from one allocation: with eight of their own the allocations took longer than
// the kernel.  (Whoever keeps one of the results keeps all of them, the table too, and a workspace of up to 12 bytes a page and 12 a sequence.)
class Words {
  public:
    explicit Words(int device) : device_(device) {}
    // Room for a result of this many words; returns where it will be.
    int64_t add(int64_t words) {
        const int64_t at = total_;
        total_ += (words + 63) & ~(int64_t)63;
        return at;
    }
    void allocate() { whole_ = at::detail::empty_cuda({total_}, at::kInt, at::Device(at::kCUDA, (c10::DeviceIndex)device_), std::nullopt); }
    int32_t* address(int64_t at) const { return static_cast<int32_t*>(whole_.mutable_data_ptr()) + at; }
    PyObject* tensor(int64_t at, at::IntArrayRef sizes) const {
        at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(whole_.storage()), whole_.key_set(), whole_.dtype());
        t.unsafeGetTensorImpl()->set_storage_offset(at);
        t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
        return THPVariable_Wrap(t);
    }

  private:
    int device_;
    int64_t total_ = 0;
    at::TensorBase whole_;
};

// A dict of results; a value that is missing (an error) leaves none.
class Results {
  public:
    Results() : dict_(PyDict_New()) {}
    ~Results() { Py_XDECREF(dict_); }
    void add(PyObject* name, PyObject* value) {
        if (!value || !dict_ || PyDict_SetItem(dict_, name, value)) Py_CLEAR(dict_);
        Py_XDECREF(value);
    }
    PyObject* take() {
        PyObject* d = dict_;
        dict_ = nullptr;
        if (!d && !PyErr_Occurred()) PyErr_NoMemory();
        return d;
    }

  private:
    PyObject* dict_;
};
struct Names {
    PyObject *refs, *page_table, *kv_len, *status, *src, *dst, *count, *accepted, *next, *tokens, *new_len;
};
const Names& names() {
    static const Names n = {PyUnicode_InternFromString("refs"), PyUnicode_InternFromString("page_table"), PyUnicode_InternFromString("kv_len"),
                            PyUnicode_InternFromString("status"), PyUnicode_InternFromString("src"), PyUnicode_InternFromString("dst"),
                            PyUnicode_InternFromString("count"), PyUnicode_InternFromString("accepted"), PyUnicode_InternFromString("next"),
                            PyUnicode_InternFromString("tokens"), PyUnicode_InternFromString("new_len")};
    return n;
}

enum { RESIZE, FORK, COMPACT };
// a: refs, page_table, kv_len, new_len or parent or None, page_size, out or None.  Error code, or the results.
PyObject* pages(int kind, PyObject* const* a) {
    const long long page_size = PyLong_AsLongLong(a[4]);
    if (PyErr_Occurred()) return nullptr;
    hos_kv_pages in, out;
    if (!state_of(a[0], a[1], a[2], page_size, -1, -1, -1, -1, &in)) return nullptr;
    const int device = THPVariable_Unpack(a[0]).get_device();
    const at::Tensor* change = nullptr;
    if (kind != COMPACT && !(change = vector(a[3], kind == RESIZE ? "new_len" : "parent", at::kInt, device, kind == RESIZE ? in.n_seq : -1))) return nullptr;
    const int64_t n_out = kind == FORK ? change->size(0) : in.n_seq, n_moves = kind == RESIZE ? in.n_seq : kind == COMPACT ? in.n_pages : 0;
    const bool given = a[5] != Py_None;
    if (given && (!PyTuple_Check(a[5]) || PyTuple_GET_SIZE(a[5]) != 3)) {
        PyErr_SetString(PyExc_TypeError, "out: expected a tuple (refs, page_table, kv_len)");
        return nullptr;
    }
    PyObject* const* o = given ? &PyTuple_GET_ITEM(a[5], 0) : nullptr;
    if (given && !state_of(o[0], o[1], o[2], page_size, device, in.n_pages, n_out, in.max_pages, &out)) return nullptr;
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
    const size_t need = kind == RESIZE ? p_resize_workspace(&in) : kind == COMPACT ? p_compact_workspace(&in) : 0;
    Words w(device);
    const int64_t scratch = w.add((int64_t)(need / 4)), status = w.add(n_out), src = w.add(n_moves), dst = w.add(n_moves), count = w.add(kind != FORK),
                  refs = w.add(given ? 0 : in.n_pages), table = w.add(given ? 0 : n_out * in.max_pages), len = w.add(given || kind == COMPACT ? 0 : n_out);
    w.allocate();
    if (!given)
        out = hos_kv_pages{in.n_pages, in.page_size, (int32_t)n_out, in.max_pages, w.address(refs), kind == COMPACT ? in.kv_len : w.address(len),
                           w.address(table), in.max_pages};
    void* st = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    const hos_kv_moves m = {w.address(src), w.address(dst), w.address(count)};
    const int rc = kind == RESIZE ? p_resize(&in, change->const_data_ptr<int32_t>(), &out, &m, w.address(status), w.address(scratch), need, st)
                 : kind == FORK ? p_fork(&in, change->const_data_ptr<int32_t>(), &out, w.address(status), st)
                                : p_compact(&in, &out, &m, w.address(status), w.address(scratch), need, st);
    if (rc) return PyLong_FromLong(rc);
    const Names& n = names();
    Results r;
    r.add(n.refs, given ? Py_NewRef(o[0]) : w.tensor(refs, {in.n_pages}));
    r.add(n.page_table, given ? Py_NewRef(o[1]) : w.tensor(table, {n_out, in.max_pages}));
    r.add(n.kv_len, kind == COMPACT ? Py_NewRef(a[2]) : given ? Py_NewRef(o[2]) : w.tensor(len, {n_out}));
    r.add(n.status, w.tensor(status, {n_out}));
    if (kind != FORK) {
        r.add(n.src, w.tensor(src, {n_moves}));
        r.add(n.dst, w.tensor(dst, {n_moves}));
        r.add(n.count, w.tensor(count, {1}));
    }
    return r.take();
}

// resize, fork, compact(refs, page_table, kv_len, new_len | parent | None, page_size, out or None)
template <int KIND> PyObject* pages_call(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* { return arity(n, 6) ? pages(KIND, a) : nullptr; });
}

// copy_pages(list of handles, list of source handles, src, dst, count or None): error code
PyObject* copy_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (!arity(n, 5)) return nullptr;
        if (!PyList_Check(a[0]) || !PyList_Check(a[1]) || PyList_GET_SIZE(a[0]) != PyList_GET_SIZE(a[1]) || PyList_GET_SIZE(a[0]) < 1) {
            PyErr_SetString(PyExc_ValueError, "as many source caches as caches, and one at least");
            return nullptr;
        }
        const Py_ssize_t layers = PyList_GET_SIZE(a[0]);
        std::vector<hos_kv_cache> to, from;
        to.reserve(layers);
        from.reserve(layers);
        const Cache* first = nullptr;
        for (Py_ssize_t l = 0; l < layers; ++l) {
            const Cache* c = cache_of(PyList_GET_ITEM(a[0], l));
            const Cache* f = c ? cache_of(PyList_GET_ITEM(a[1], l)) : nullptr;
            if (!f) return nullptr;
            if (!first) first = c;
            for (const Cache* x : {c, f})
                if (x->device != first->device) {
                    PyErr_SetString(PyExc_ValueError, "the caches must be on one device");
                    return nullptr;
                }
            for (const Cache* x : {c, f})
                if (x->c.n_kv_heads != first->c.n_kv_heads || x->c.page_size != first->c.page_size || x->c.head_dim != first->c.head_dim ||
                    x->c.type != first->c.type || x->c.format != first->c.format) {
                    PyErr_SetString(PyExc_ValueError, "the caches must have the same heads, page size, head_dim, dtype and format");
                    return nullptr;
                }
            to.push_back(c->c);
            from.push_back(f->c);
        }
        for (Py_ssize_t l = 0; l < layers; ++l)
            if (to[l].n_pages != to[0].n_pages || from[l].n_pages != from[0].n_pages) {
                PyErr_SetString(PyExc_ValueError, "all layers must have the same number of pages");
                return nullptr;
            }
        const at::Tensor* src = vector(a[2], "src", at::kInt, first->device, -1);
        const at::Tensor* dst = src ? vector(a[3], "dst", at::kInt, first->device, src->size(0)) : nullptr;
        if (!dst) return nullptr;
        const at::Tensor* count = nullptr;
        if (a[4] != Py_None && !(count = vector(a[4], "count", at::kInt, first->device, 1))) return nullptr;
        if (src->size(0) > first->status.numel()) return PyLong_FromLong(STATUS_TOO_SHORT);
        const c10::cuda::CUDAGuard guard(first->device);
        const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream(first->device);
        return PyLong_FromLong(p_copy_pages(to.data(), from.data(), (int)layers, src->const_data_ptr<int32_t>(), dst->const_data_ptr<int32_t>(),
                                            count ? count->const_data_ptr<int32_t>() : nullptr, (int)src->size(0), first->words(st), st.stream()));
    });
}

// A [n_tokens][vocab] tensor of probabilities.
const at::Tensor* probabilities(PyObject* o, const char* what, const at::Tensor* like) {
    const at::Tensor* t = tensor(o, what);
    if (!t) return nullptr;
    const at::ScalarType k = t->scalar_type();
    if (!t->is_cuda() || (k != at::kFloat && k != at::kHalf && k != at::kBFloat16) ||
        (like && (k != like->scalar_type() || t->get_device() != like->get_device()))) {
        PyErr_Format(PyExc_TypeError, like ? "%s: expected a tensor of target's dtype on its device" : "%s: expected a CUDA tensor of float32, float16 or bfloat16", what);
        return nullptr;
    }
    if (t->dim() != 2 || t->size(1) < 1 || (t->size(1) > 1 && t->stride(1) != 1) || (like && t->sizes() != like->sizes())) {
        PyErr_Format(PyExc_ValueError, "%s: expected [n_tokens][vocab] with dense rows", what);
        return nullptr;
    }
    if (t->size(0) > INT32_MAX || t->size(1) > INT32_MAX) {
        PyErr_SetString(PyExc_ValueError, "sizes beyond 32 bits");
        return nullptr;
    }
    if (t->requires_grad() && c10::GradMode::is_enabled()) {
        PyErr_Format(PyExc_ValueError, "%s requires grad, and there is no backward pass: detach it, or call under torch.no_grad()", what);
        return nullptr;
    }
    return t;
}

// verify(tokens, target, draft or None, tok_off, u_accept, u_sample, kv_len or None): error code, or the results
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (!arity(n, 7)) return nullptr;
        const at::Tensor* target = probabilities(a[1], "target", nullptr);
        if (!target) return nullptr;
        const at::Tensor* draft = nullptr;
        if (a[2] != Py_None && !(draft = probabilities(a[2], "draft", target))) return nullptr;
        const int device = target->get_device();
        const int64_t n_tok = target->size(0);
        const at::Tensor* tokens = vector(a[0], "tokens", at::kInt, device, n_tok);
        const at::Tensor* off = tokens ? vector(a[3], "tok_off", at::kInt, device, -1) : nullptr;
        if (!off) return nullptr;
        if (off->size(0) < 1) {
            PyErr_SetString(PyExc_ValueError, "tok_off must have n_seq + 1 entries");
            return nullptr;
        }
        const int64_t n_seq = off->size(0) - 1;
        const at::Tensor* ua = vector(a[4], "u_accept", at::kFloat, device, n_tok);
        const at::Tensor* us = ua ? vector(a[5], "u_sample", at::kFloat, device, n_seq) : nullptr;
        if (!us) return nullptr;
        const at::Tensor* len = nullptr;
        if (a[6] != Py_None && !(len = vector(a[6], "kv_len", at::kInt, device, n_seq))) return nullptr;
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
        Words w(device);
        const int64_t accepted = w.add(n_seq), next = w.add(n_seq), out = w.add(n_tok), status = w.add(n_seq), now = w.add(len ? n_seq : 0);
        w.allocate();
        hos_drafts d = {};
        d.n_seq = (int32_t)n_seq;
        d.n_tokens = (int32_t)n_tok;
        d.vocab = (int32_t)target->size(1);
        d.type = target->scalar_type() == at::kFloat ? HOS_TYPE_FP32 : target->scalar_type() == at::kHalf ? HOS_TYPE_FP16 : HOS_TYPE_BF16;
        d.tok_off = off->const_data_ptr<int32_t>();
        d.tokens = tokens->const_data_ptr<int32_t>();
        d.target = target->const_data_ptr();
        d.target_stride = n_tok > 1 ? target->stride(0) : d.vocab;
        if (draft) {
            d.draft = draft->const_data_ptr();
            d.draft_stride = n_tok > 1 ? draft->stride(0) : d.vocab;
        }
        d.u_accept = ua->const_data_ptr<float>();
        d.u_sample = us->const_data_ptr<float>();
        d.accepted = w.address(accepted);
        d.next = w.address(next);
        d.out_tokens = w.address(out);
        d.status = w.address(status);
        if (len) {
            d.kv_len = len->const_data_ptr<int32_t>();
            d.new_len = w.address(now);
        }
        const int rc = p_verify(&d, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream());
        if (rc) return PyLong_FromLong(rc);
        const Names& name = names();
        Results r;
        r.add(name.accepted, w.tensor(accepted, {n_seq}));
        r.add(name.next, w.tensor(next, {n_seq}));
        r.add(name.tokens, w.tensor(out, {n_tok}));
        r.add(name.new_len, len ? w.tensor(now, {n_seq}) : Py_NewRef(Py_None));
        r.add(name.status, w.tensor(status, {n_seq}));
        return r.take();
    });
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"init", FAST(init)}, {"cache", FAST(cache)}, {"set_status", FAST(set_status)}, {"append", FAST(append)},
                         {"read", FAST(read)}, {"attention", FAST(attention)}, {"resize", FAST(pages_call<RESIZE>)},
                         {"fork", FAST(pages_call<FORK>)}, {"compact", FAST(pages_call<COMPACT>)}, {"copy_pages", FAST(copy_pages)},
                         {"verify", FAST(verify)}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv() { return PyModule_Create(&module); }
