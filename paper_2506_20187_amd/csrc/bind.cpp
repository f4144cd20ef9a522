// Native argument marshalling for the entry points of a decode step.
//
// A decode step of a small batch is two launches of 5-15 us each.  Through ctypes (a property, a method call
// and a c_void_p object per tensor, and torch.cuda.current_stream()) the host took 8.0 us per call of chunk_score,
// launch included, and 24.5 us for the two calls of the fp32 4K step (three launches then), so the host, not the
// GPU, set the pace of such a step.  Here a tensor costs one type check and three field reads: 4.0 us per
// chunk_score, 9.0 us per step (two launches).
//
// Every function takes the arguments of the C entry point of the same name (include/leoam.h) in its
// order, tensors or None for device pointers, the stream as whatever binding._stream takes (it is called
// last, after every tensor has been looked at), and returns the status.  Nothing is kept from one call for
// the next: every tensor is looked at on every call.  Only plain torch.Tensor objects are read here; anything
// else (subclasses, other objects with the same methods, tensors whose fields raise) goes through the checker
// that binding.py registers, which raises what it always raised.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/leoam.h"

namespace {

PyObject* g_shape_type = nullptr;      // binding.Shape
PyObject* g_pages_type = nullptr;      // binding.Pages
PyObject* g_pointer_of = nullptr;      // binding._p: tensor -> ctypes.c_void_p or None, raises ValueError

PyObject* g_stream_of = nullptr;       // binding._stream: stream object, integer or None -> handle

// the entry points of the library that binding.py loaded (addresses handed over by setup, so this
// module depends on no second copy of it)
struct {
    decltype(&::chunk_score) chunk_score;
    decltype(&::chunk_score_pin) chunk_score_pin;
    decltype(&::kv_chunk_abstract_append) kv_chunk_abstract_append;
    decltype(&::chunk_topk_select) chunk_topk_select;
    decltype(&::sparse_chunk_attention_decode) sparse_chunk_attention_decode;
    decltype(&::chunk_select_attention_decode) chunk_select_attention_decode;
    decltype(&::kv_page_append) kv_page_append;
    decltype(&::page_attention_decode) page_attention_decode;
    decltype(&::page_attention_prefill) page_attention_prefill;
} g_lib;
constexpr int kEntryPoints = 9;
static_assert(sizeof(g_lib) == kEntryPoints * sizeof(void*), "one address each");

// device pointer of a tensor (or None); false with a Python error set
bool pointer_arg(PyObject* o, void** out) {
    *out = nullptr;
    if (o == Py_None) return true;
    if (THPVariable_CheckExact(o)) {
        try {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (t.is_cuda() && t.is_contiguous()) {
                *out = t.data_ptr();
                return true;
            }
        } catch (const std::exception&) {
            // (the checker below raises it as the Python error it is)
        }
    }
    PyObject* p = PyObject_CallOneArg(g_pointer_of, o);
    if (!p) return false;
    PyObject* v = p == Py_None ? Py_NewRef(Py_None) : PyObject_GetAttrString(p, "value");
    Py_DECREF(p);
    if (!v) return false;
    if (v != Py_None) *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}

// 32-bit integers wrap as ctypes lets them
bool int_arg(PyObject* o, int32_t* out) {
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) return false;
    *out = (int32_t)(uint32_t)v;
    return true;
}

// the C struct that a ctypes Structure of type `type` holds
template <typename S> bool struct_arg(PyObject* o, PyObject* type, const char* name, S* out) {
    const int is = PyObject_IsInstance(o, type);
    if (is < 0) return false;
    if (is == 0) {
        PyErr_Format(PyExc_TypeError, "expected a %s", name);
        return false;
    }
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return false;
    const bool ok = view.len == (Py_ssize_t)sizeof(S);
    if (ok) memcpy(out, view.buf, sizeof(S));
    else PyErr_Format(PyExc_TypeError, "%s has another layout", name);
    PyBuffer_Release(&view);
    return ok;
}

// The arguments of one call, read in order; `ok` turns false (with a Python error set) at the first bad one.
struct Args {
    PyObject* const* a;
    Py_ssize_t n, i = 0;
    bool ok = true;
    leoam_shape shape;
    leoam_pages pages;
    int device = -1;      // the current device, once `tensor` has asked for it

    Args(PyObject* const* args, Py_ssize_t nargs, Py_ssize_t wanted, bool paged = false) : a(args), n(nargs) {
        if (nargs != wanted) {
            PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", wanted, nargs);
            ok = false;
            return;
        }
        ok = paged ? struct_arg(a[0], g_pages_type, "Pages", &pages) : struct_arg(a[0], g_shape_type, "Shape", &shape);
        i = 1;
    }

    // ---- arguments of the paged cache's calls: a tensor's type, device and size are looked at ----
    bool refuse(const char* name, const char* why) {
        PyErr_Format(PyExc_ValueError, "%s: %s", name, why);
        return ok = false;
    }
    const at::Tensor* tensor(const char* name, at::ScalarType type, bool nullable) {
        if (!ok) return nullptr;
        PyObject* o = a[i++];
        if (o == Py_None) {
            if (!nullable) refuse(name, "expected a tensor");
            return nullptr;
        }
        if (!THPVariable_Check(o)) {
            refuse(name, "expected a tensor");
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda()) refuse(name, "expected a CUDA tensor");
        else if (t.scalar_type() != type) refuse(name, "another element type than the call wants");
        else if (t.get_device() != here()) refuse(name, "on another device than the current one");
        return ok ? &t : nullptr;
    }
    int here() {
        if (device < 0) device = (int)c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index();
        return device;
    }
    // contiguous, with at least `elements` elements
    template <typename P = void> P* buffer(const char* name, at::ScalarType type, int64_t elements, bool nullable = false) {
        try {
            const at::Tensor* t = tensor(name, type, nullable);
            if (!t) return nullptr;
            if (!t->is_contiguous()) refuse(name, "expected a contiguous tensor");
            else if (t->numel() < elements) refuse(name, "fewer elements than the call needs");
            return ok ? static_cast<P*>(t->data_ptr()) : nullptr;
        } catch (const std::exception& e) {
            refuse(name, e.what());
            return nullptr;
        }
    }
    // rows [n, heads, 128], each contiguous; *rows = n (or must be it, if it is not negative)
    void* strided_rows(const char* name, at::ScalarType type, int64_t heads, int64_t* rows, int64_t* stride, bool nullable = false) {
        *stride = 0;
        try {
            const at::Tensor* t = tensor(name, type, nullable);
            if (!t) return nullptr;
            if (t->dim() != 3 || t->size(1) != heads || t->size(2) != 128) refuse(name, "expected [rows, heads, 128]");
            else if (*rows >= 0 && t->size(0) != *rows) refuse(name, "another number of rows than the others");
            else if (t->stride(2) != 1 || (heads > 1 && t->stride(1) != 128)) refuse(name, "the heads of a row must be contiguous");
            if (!ok) return nullptr;
            *rows = t->size(0);
            *stride = t->stride(0);
            return t->data_ptr();
        } catch (const std::exception& e) {
            refuse(name, e.what());
            return nullptr;
        }
    }
    // bytes of a workspace tensor of any type
    void* scratch(const char* name, size_t* bytes) {
        *bytes = 0;
        if (!ok) return nullptr;
        PyObject* o = a[i++];
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) {
            refuse(name, "expected a tensor");
            return nullptr;
        }
        try {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (!t.is_cuda() || !t.is_contiguous()) refuse(name, "expected a contiguous CUDA tensor");
            else if (t.get_device() != here()) refuse(name, "on another device than the current one");
            if (!ok) return nullptr;
            *bytes = t.numel() * t.element_size();
            return t.data_ptr();
        } catch (const std::exception& e) {
            refuse(name, e.what());
            return nullptr;
        }
    }
    at::ScalarType type_of(int32_t tag) const {
        switch (tag) {
        case LEOAM_F32: return at::kFloat;
        case LEOAM_F16: return at::kHalf;
        case LEOAM_BF16: return at::kBFloat16;
        default: return at::kFloat8_e4m3fn;
        }
    }
    template <typename P = void> P* ptr() {
        void* p = nullptr;
        if (ok) ok = pointer_arg(a[i++], &p);
        return static_cast<P*>(p);
    }
    int32_t i32() {
        int32_t v = 0;
        if (ok) ok = int_arg(a[i++], &v);
        return v;
    }
    float f32() {
        double v = 0.0;
        if (ok) {
            v = PyFloat_AsDouble(a[i++]);
            ok = !(v == -1.0 && PyErr_Occurred());
        }
        return (float)v;
    }
    size_t bytes() {
        size_t v = 0;
        if (ok) {
            v = PyLong_AsSize_t(a[i++]);
            ok = !(v == (size_t)-1 && PyErr_Occurred());
        }
        return v;
    }
    void* stream() {
        void* v = nullptr;
        if (ok) {
            PyObject* s = PyObject_CallOneArg(g_stream_of, a[i++]);
            if (s) v = PyLong_AsVoidPtr(s);
            Py_XDECREF(s);
            ok = !PyErr_Occurred();
        }
        return v;
    }
};

// the call runs without the interpreter lock (a launch can wait for room in the queue)
template <typename F> PyObject* status_of(const Args& args, F&& call) {
    if (!args.ok) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

PyObject* py_setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4 + kEntryPoints) {
        PyErr_SetString(PyExc_TypeError, "setup(shape_type, pages_type, pointer_of, stream_of, addresses in the order of g_lib)");
        return nullptr;
    }
    void* at[kEntryPoints];
    for (int i = 0; i < kEntryPoints; ++i) {
        at[i] = PyLong_AsVoidPtr(a[4 + i]);
        if (PyErr_Occurred()) return nullptr;
    }
    memcpy(&g_lib, at, sizeof(g_lib));
    Py_XDECREF(g_shape_type);
    Py_XDECREF(g_pages_type);
    Py_XDECREF(g_pointer_of);
    Py_XDECREF(g_stream_of);
    g_shape_type = Py_NewRef(a[0]);
    g_pages_type = Py_NewRef(a[1]);
    g_pointer_of = Py_NewRef(a[2]);
    g_stream_of = Py_NewRef(a[3]);
    Py_RETURN_NONE;
}

PyObject* py_chunk_score(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Args r(a, n, 7);
    const void* q = r.ptr();
    const void* abstract = r.ptr();
    const int32_t* n_chunks = r.ptr<int32_t>();
    float* ub = r.ptr<float>();
    float* lb = r.ptr<float>();
    void* st = r.stream();
    return status_of(r, [&] { return g_lib.chunk_score(&r.shape, q, abstract, n_chunks, ub, lb, st); });
}

PyObject* py_chunk_score_pin(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Args r(a, n, 6);
    const int32_t* n_chunks = r.ptr<int32_t>();
    const int32_t sink = r.i32(), tail = r.i32();
    float* ub = r.ptr<float>();
    void* st = r.stream();
    return status_of(r, [&] { return g_lib.chunk_score_pin(&r.shape, n_chunks, sink, tail, ub, st); });
}

PyObject* py_abstract_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Args r(a, n, 8);
    const void* K = r.ptr();
    int32_t* off = r.ptr<int32_t>();
    int32_t* n_chunks = r.ptr<int32_t>();
    const int32_t chunk_size = r.i32();
    void* abstract = r.ptr();
    int32_t* status = r.ptr<int32_t>();
    void* st = r.stream();
    return status_of(r, [&] { return g_lib.kv_chunk_abstract_append(&r.shape, K, off, n_chunks, chunk_size, abstract, status, st); });
}

PyObject* py_topk_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Args r(a, n, 12);
    const float* ub = r.ptr<float>();
    const int32_t* off = r.ptr<int32_t>();
    const int32_t* n_chunks = r.ptr<int32_t>();
    const int32_t max_chunks = r.i32(), budget = r.i32();
    int32_t* idx = r.ptr<int32_t>();
    int32_t* count = r.ptr<int32_t>();
    int32_t* tokens = r.ptr<int32_t>();
    void* ws = r.ptr();
    const size_t ws_bytes = r.bytes();
    void* st = r.stream();
    return status_of(r, [&] {
        return g_lib.chunk_topk_select(&r.shape, ub, off, n_chunks, max_chunks, budget, idx, count, tokens, ws, ws_bytes, st);
    });
}

PyObject* py_sparse_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Args r(a, n, 15);
    const void* q = r.ptr();
    const void* K = r.ptr();
    const void* V = r.ptr();
    const void* qmeta = r.ptr();
    const int32_t* off = r.ptr<int32_t>();
    const int32_t* n_chunks = r.ptr<int32_t>();
    const int32_t* idx = r.ptr<int32_t>();
    const int32_t* count = r.ptr<int32_t>();
    const float scale = r.f32();
    float* out = r.ptr<float>();
    float* lse = r.ptr<float>();
    void* ws = r.ptr();
    const size_t ws_bytes = r.bytes();
    void* st = r.stream();
    return status_of(r, [&] {
        return g_lib.sparse_chunk_attention_decode(&r.shape, q, K, V, qmeta, off, n_chunks, idx, count, scale, out, lse, ws, ws_bytes, st);
    });
}

PyObject* py_select_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Args r(a, n, 19);
    const float* ub = r.ptr<float>();
    const void* q = r.ptr();
    const void* K = r.ptr();
    const void* V = r.ptr();
    const void* qmeta = r.ptr();
    const int32_t* off = r.ptr<int32_t>();
    const int32_t* n_chunks = r.ptr<int32_t>();
    const int32_t max_chunks = r.i32(), budget = r.i32();
    const float scale = r.f32();
    int32_t* idx = r.ptr<int32_t>();
    int32_t* count = r.ptr<int32_t>();
    int32_t* tokens = r.ptr<int32_t>();
    float* out = r.ptr<float>();
    float* lse = r.ptr<float>();
    void* ws = r.ptr();
    const size_t ws_bytes = r.bytes();
    void* st = r.stream();
    return status_of(r, [&] {
        return g_lib.chunk_select_attention_decode(&r.shape, ub, q, K, V, qmeta, off, n_chunks, max_chunks, budget, scale, idx, count,
                                             tokens, out, lse, ws, ws_bytes, st);
    });
}

// The pages of the pool and what finds them: k_pages, v_pages, k_scale, v_scale, page_table are arguments of all three calls,
// in this order but for what stands between.
struct Pool {
    void *k, *v;
    float *ks, *vs;
    int64_t elements, scales;
    at::ScalarType kv, row;
    explicit Pool(const Args& r) {
        const leoam_pages& p = r.pages;
        elements = (int64_t)p.n_pages * p.n_kv_heads * p.page_size * p.head_dim;
        scales = (int64_t)p.n_pages * p.n_kv_heads;
        kv = r.type_of(p.kv_dtype);
        row = r.type_of(p.q_dtype);
    }
    void read(Args& r) {
        k = r.buffer("k_pages", kv, elements);
        v = r.buffer("v_pages", kv, elements);
        ks = r.buffer<float>("k_scale", at::kFloat, scales, kv != at::kFloat8_e4m3fn);
        vs = r.buffer<float>("v_scale", at::kFloat, scales, kv != at::kFloat8_e4m3fn);
    }
};

// rows of a call fit its 32-bit counts
bool rows_fit(Args& r, int64_t rows) { return !r.ok || rows <= 0x7fffffff || r.refuse("rows", "more than 2^31 - 1"); }

PyObject* py_page_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Args r(a, n, 18, true);
    if (!r.ok) return nullptr;
    const leoam_pages& s = r.pages;
    Pool pool(r);
    int64_t q_rows = -1, rows = -1, q_stride, k_stride, v_stride;
    const void* q = r.strided_rows("q", pool.row, s.n_q_heads, &q_rows, &q_stride, true);
    if (q_rows >= 0) rows = q_rows;
    const void* k = r.strided_rows("k", pool.row, s.n_kv_heads, &rows, &k_stride);
    const void* v = r.strided_rows("v", pool.row, s.n_kv_heads, &rows, &v_stride);
    rows_fit(r, rows);
    const int32_t* new_off = r.buffer<int32_t>("new_off", at::kInt, (int64_t)s.batch + 1, true);
    const int32_t* len = r.buffer<int32_t>("seq_len", at::kInt, s.batch);
    const int32_t* table = r.buffer<int32_t>("page_table", at::kInt, (int64_t)s.batch * s.max_pages);
    const float* rope = r.buffer<float>("rope", at::kFloat, (int64_t)s.rope_len * s.rot_dim, s.rot_dim == 0);
    void* q_out = r.buffer("q_out", pool.row, q_rows * s.n_q_heads * s.head_dim, true);
    pool.read(r);
    void* abstract = r.buffer("abstract", pool.row, (int64_t)s.batch * s.n_kv_heads * s.max_pages * 2 * s.head_dim, true);
    int32_t* off = r.buffer<int32_t>("chunk_off", at::kInt, (int64_t)s.batch * (s.max_pages + 1), true);
    int32_t* n_chunks = r.buffer<int32_t>("n_chunks", at::kInt, s.batch, true);
    int32_t* status = r.buffer<int32_t>("status", at::kInt, s.batch, true);
    void* st = r.stream();
    return status_of(r, [&] {
        return g_lib.kv_page_append(&s, q, q_stride, k, k_stride, v, v_stride, (int32_t)rows, new_off, len, table, rope, q_out,
                                    pool.k, pool.v, pool.ks, pool.vs, abstract, off, n_chunks, status, st);
    });
}

PyObject* py_page_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Args r(a, n, 15, true);
    if (!r.ok) return nullptr;
    const leoam_pages& s = r.pages;
    Pool pool(r);
    const int64_t heads = (int64_t)s.batch * s.n_q_heads;
    const void* q = r.buffer("q", pool.row, heads * s.head_dim);
    pool.read(r);
    const int32_t* table = r.buffer<int32_t>("page_table", at::kInt, (int64_t)s.batch * s.max_pages);
    const int32_t* len = r.buffer<int32_t>("seq_len", at::kInt, s.batch);
    int32_t k_max = 0;
    const int32_t* idx = nullptr;
    try {
        const at::Tensor* t = r.tensor("sel_idx", at::kInt, true);
        if (t) {
            if (t->dim() != 3 || t->size(0) != s.batch || t->size(1) != s.n_kv_heads || t->size(2) > 0x7fffffff)
                r.refuse("sel_idx", "expected [batch, n_kv_heads, k_max]");
            else if (!t->is_contiguous()) r.refuse("sel_idx", "expected a contiguous tensor");
            else {
                k_max = (int32_t)t->size(2);
                idx = static_cast<const int32_t*>(t->data_ptr());
            }
        }
    } catch (const std::exception& e) {
        r.refuse("sel_idx", e.what());
    }
    const int32_t* count = r.buffer<int32_t>("sel_count", at::kInt, (int64_t)s.batch * s.n_kv_heads, true);
    const float scale = r.f32();
    float* out = r.buffer<float>("out", at::kFloat, heads * s.head_dim);
    float* lse = r.buffer<float>("lse", at::kFloat, heads, true);
    size_t bytes;
    void* ws = r.scratch("workspace", &bytes);
    void* st = r.stream();
    return status_of(r, [&] {
        return g_lib.page_attention_decode(&s, q, pool.k, pool.v, pool.ks, pool.vs, table, len, idx, count, k_max, scale, out, lse, ws,
                                           bytes, st);
    });
}

PyObject* py_page_prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Args r(a, n, 14, true);
    if (!r.ok) return nullptr;
    const leoam_pages& s = r.pages;
    Pool pool(r);
    int64_t rows = -1, stride;
    const void* q = r.strided_rows("q", pool.row, s.n_q_heads, &rows, &stride);
    rows_fit(r, rows);
    if (r.ok && rows > 1 && stride != (int64_t)s.n_q_heads * s.head_dim) r.refuse("q", "expected a contiguous tensor");
    const int32_t* new_off = r.buffer<int32_t>("new_off", at::kInt, (int64_t)s.batch + 1, true);
    pool.read(r);
    const int32_t* table = r.buffer<int32_t>("page_table", at::kInt, (int64_t)s.batch * s.max_pages);
    const int32_t* len = r.buffer<int32_t>("seq_len", at::kInt, s.batch);
    const float scale = r.f32();
    void* out = r.buffer("out", pool.row, rows * s.n_q_heads * s.head_dim);
    float* lse = r.buffer<float>("lse", at::kFloat, rows * s.n_q_heads, true);
    size_t bytes;
    void* ws = r.scratch("workspace", &bytes);
    void* st = r.stream();
    return status_of(r, [&] {
        return g_lib.page_attention_prefill(&s, q, (int32_t)rows, new_off, pool.k, pool.v, pool.ks, pool.vs, table, len, scale, out, lse,
                                            ws, bytes, st);
    });
}

#define LEOAM_METHOD(name, fn) {name, (PyCFunction)(void (*)(void))fn, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {LEOAM_METHOD("setup", py_setup),
                           LEOAM_METHOD("chunk_score", py_chunk_score),
                           LEOAM_METHOD("chunk_score_pin", py_chunk_score_pin),
                           LEOAM_METHOD("kv_chunk_abstract_append", py_abstract_append),
                           LEOAM_METHOD("chunk_topk_select", py_topk_select),
                           LEOAM_METHOD("sparse_chunk_attention_decode", py_sparse_attention),
                           LEOAM_METHOD("chunk_select_attention_decode", py_select_attention),
                           LEOAM_METHOD("kv_page_append", py_page_append),
                           LEOAM_METHOD("page_attention_decode", py_page_decode),
                           LEOAM_METHOD("page_attention_prefill", py_page_prefill),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bind() { return PyModule_Create(&g_module); }
