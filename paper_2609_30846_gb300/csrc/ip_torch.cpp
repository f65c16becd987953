// Short forms of the Python calls with run-time scales and on the 4-bit cache, for their usual
// arguments: plain contiguous tensors (or matrices) of the current device, its current stream.
// Each makes the checks of the general form in place, allocates the outputs and calls the C
// entry point; it returns the outputs, the entry point's error code, or None for arguments that
// the general form (Python, over ctypes) has to look at.  A decoder's single-token calls are
// shorter on the GPU than this work takes in Python.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "ip_mhsa.h"

namespace {

// The entry points of the library that Python has loaded.
struct Entries {
    decltype(&ip_quantize_rows_i8) quantize;
    decltype(&ip_linear_scaled_i8) linear;
    decltype(&ip_kv4_append) append;
    decltype(&ip_kv4_read) read;
    decltype(&ip_kv4_attention) attention;
} g_entry;

constexpr int64_t ROW_BYTES = 144;

int code_of(at::ScalarType t) {
    return t == at::kFloat ? IP_F32 : (t == at::kHalf ? IP_F16 : (t == at::kBFloat16 ? IP_BF16 : -1));
}

// The tensor behind o, nullptr if o is none or not a strided one on CUDA.
const at::Tensor *tensor(PyObject *o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}
bool contiguous(const at::Tensor *t, at::ScalarType type, int dev) {
    return t && t->scalar_type() == type && t->get_device() == dev && t->is_contiguous();
}
bool vector(const at::Tensor *t, at::ScalarType type, int64_t n, int dev) {
    return contiguous(t, type, dev) && t->dim() == 1 && t->size(0) == n;
}
// None or a tensor: false for what is neither; p is its data.
bool maybe_vector(PyObject *o, at::ScalarType type, int64_t n, int dev, const void *&p) {
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = tensor(o);
    if (!vector(t, type, n, dev)) return false;
    p = t->const_data_ptr();
    return true;
}
bool fits(int64_t n) { return n <= INT_MAX; }

ip_stream_t stream_of(int dev) {
    return reinterpret_cast<ip_stream_t>(c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(dev)).stream());
}
at::Tensor empty(at::IntArrayRef shape, const at::Tensor &like, at::ScalarType type) {
    return at::empty(shape, like.options().dtype(type).requires_grad(false));
}
// The caller's output o, or a new one for None; false for what the general form has to look at.
bool output(PyObject *o, at::IntArrayRef shape, const at::Tensor &like, at::ScalarType type, at::Tensor &out) {
    if (o == Py_None) {
        out = empty(shape, like, type);
        return true;
    }
    const at::Tensor *t = tensor(o);
    if (!contiguous(t, type, like.get_device()) || t->sizes() != shape) return false;
    out = *t;
    return true;
}

// Calls without the interpreter's lock: a launch may wait for room in its stream's queue.
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }      // before an exception becomes Python's too
};
template <typename F>
int unlocked(F &&f) {
    const Unlocked u;
    return f();
}

PyObject *pair(const at::Tensor &a, const at::Tensor &b) {
    PyObject *x = THPVariable_Wrap(a), *y = x ? THPVariable_Wrap(b) : nullptr;
    PyObject *r = y ? PyTuple_New(2) : nullptr;
    if (!r) {
        Py_XDECREF(x);
        Py_XDECREF(y);
        return nullptr;
    }
    PyTuple_SET_ITEM(r, 0, x);
    PyTuple_SET_ITEM(r, 1, y);
    return r;
}

bool arity(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, n);
    return false;
}

// (x, q, scale)
PyObject *quantize_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 3)) return nullptr;
    const at::Tensor *x = tensor(a[0]);
    if (!x || x->dim() < 1 || !x->is_contiguous()) Py_RETURN_NONE;
    const int dev = x->get_device(), code = code_of(x->scalar_type());
    const int64_t d = x->size(-1);
    if (code < 0 || d < 1 || !fits(d) || dev != c10::cuda::current_device()) Py_RETURN_NONE;
    c10::SmallVector<int64_t, 6> shape(x->sizes().begin(), x->sizes().end());
    int64_t ld = (d + 15) / 16 * 16;
    at::Tensor q, scale;
    if (a[1] != Py_None || ld == d) {
        if (!output(a[1], shape, *x, at::kChar, q)) Py_RETURN_NONE;
        ld = d;
    } else {
        c10::SmallVector<int64_t, 6> strides(shape.size(), 1);
        int64_t step = ld;
        for (size_t i = shape.size() - 1; i-- > 0; step *= shape[i] > 1 ? shape[i] : 1) strides[i] = step;
        q = at::empty_strided(shape, strides, x->options().dtype(at::kChar).requires_grad(false));
    }
    shape.pop_back();
    if (!output(a[2], shape, *x, at::kFloat, scale)) Py_RETURN_NONE;
    const int rc = unlocked([&] {
        return g_entry.quantize(x->const_data_ptr(), code, x->numel() / d, static_cast<int>(d), d,
                                static_cast<int8_t *>(q.data_ptr()), ld, static_cast<float *>(scale.data_ptr()),
                                stream_of(dev));
    });
    if (rc != IP_OK) return PyLong_FromLong(rc);
    return pair(q, scale);
    END_HANDLE_TH_ERRORS
}

// Row stride of a matrix or a contiguous tensor, 0 for what the general form has to look at.
int64_t row_stride(const at::Tensor &t) {
    if (t.stride(-1) != 1 && t.size(-1) != 1) return 0;      // one row too: its elements are read as consecutive
    if (t.numel() == t.size(-1)) return (t.size(-1) + 15) / 16 * 16;      // one row: any stride does
    if (t.is_contiguous()) return t.size(-1);
    return t.dim() == 2 && t.stride(1) == 1 ? t.stride(0) : 0;
}

// (x, sx, w, sw, bias, act, dtype, out, workspace)
PyObject *linear_scaled(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 9)) return nullptr;
    const at::Tensor *x = tensor(a[0]), *sx = tensor(a[1]), *w = tensor(a[2]), *ws = tensor(a[8]);
    if (!x || !sx || !w || !ws || !PyLong_CheckExact(a[5])) Py_RETURN_NONE;
    at::ScalarType type = at::kBFloat16;
    if (THPDtype_Check(a[6])) type = reinterpret_cast<THPDtype *>(a[6])->scalar_type;
    else if (a[6] != Py_None) Py_RETURN_NONE;
    else if (THPVariable_CheckExact(a[7])) type = THPVariable_Unpack(a[7]).scalar_type();
    const int dev = x->get_device(), code = code_of(type);
    if (code < 0 || dev != c10::cuda::current_device() || x->dim() < 1 || x->scalar_type() != at::kChar ||
        w->dim() != 2 || w->scalar_type() != at::kChar || w->get_device() != dev || !contiguous(sx, at::kFloat, dev) ||
        !contiguous(ws, at::kByte, dev))
        Py_RETURN_NONE;
    const int64_t N = w->size(0), K = w->size(1);
    const long act = PyLong_AsLong(a[5]);
    if (PyErr_Occurred()) PyErr_Clear();
    if (K < 1 || N < 1 || !fits(N) || !fits(K) || x->size(-1) != K || act < 0 || act > INT_MAX) Py_RETURN_NONE;
    const int64_t ldx = row_stride(*x), ldw = row_stride(*w);
    const at::IntArrayRef lead = x->sizes().slice(0, x->dim() - 1);
    const void *sw, *bias;
    if (ldx < K || ldw < K || (ldx | ldw) % 16 != 0 || sx->sizes() != lead ||
        !maybe_vector(a[3], at::kFloat, N, dev, sw) || !sw || !maybe_vector(a[4], at::kFloat, N, dev, bias))
        Py_RETURN_NONE;
    c10::SmallVector<int64_t, 6> shape(lead.begin(), lead.end());
    shape.push_back(N);
    at::Tensor out;
    if (!output(a[7], shape, *x, type, out)) Py_RETURN_NONE;
    const int rc = unlocked([&] {
        return g_entry.linear(static_cast<const int8_t *>(x->const_data_ptr()), ldx,
                              static_cast<const float *>(sx->const_data_ptr()),
                              static_cast<const int8_t *>(w->const_data_ptr()), ldw, static_cast<const float *>(sw),
                              static_cast<const float *>(bias), static_cast<int>(act), x->numel() / K,
                              static_cast<int>(K), static_cast<int>(N), out.data_ptr(), N, code, ws->data_ptr(),
                              static_cast<size_t>(ws->numel()), stream_of(dev));
    });
    return rc == IP_OK ? THPVariable_Wrap(out) : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// A cache with its table, a workspace and two int32 vectors (the second may be None).
struct Cache {
    int n_pages, heads, page, width;
    const int32_t *table, *first, *second;
    void *pages, *ws;
    size_t ws_bytes;

    bool take(int dev, int64_t B, PyObject *po_cache, PyObject *po_table, PyObject *po_first, PyObject *po_second,
              PyObject *po_ws) {
        const at::Tensor *c = tensor(po_cache), *t = tensor(po_table), *f = tensor(po_first), *w = tensor(po_ws);
        const void *s;
        if (dev != c10::cuda::current_device() || !contiguous(c, at::kByte, dev) || !contiguous(t, at::kInt, dev) ||
            !contiguous(w, at::kByte, dev) || c->dim() != 3 || c->size(2) % ROW_BYTES != 0 || t->dim() != 2 ||
            t->size(0) != B || !vector(f, at::kInt, B, dev) || !maybe_vector(po_second, at::kInt, B, dev, s) ||
            !fits(c->size(0)) || !fits(c->size(1)) || !fits(c->size(2)) || !fits(t->size(1)) || !fits(B))
            return false;
        n_pages = static_cast<int>(c->size(0));
        heads = static_cast<int>(c->size(1));
        page = static_cast<int>(c->size(2) / ROW_BYTES);
        width = static_cast<int>(t->size(1));
        table = static_cast<const int32_t *>(t->const_data_ptr());
        first = static_cast<const int32_t *>(f->const_data_ptr());
        second = static_cast<const int32_t *>(s);
        pages = c->data_ptr();
        ws = w->data_ptr();
        ws_bytes = static_cast<size_t>(w->numel());
        return true;
    }
};

// [B, T, H, 128] with contiguous channels; st: the other axes' strides.
bool rows_of_heads(const at::Tensor *t, long long (&st)[3]) {
    if (!t || t->dim() != 4 || t->size(3) != IP_DH || t->stride(3) != 1 || !fits(t->size(0)) || !fits(t->size(1)) ||
        !fits(t->size(2)))
        return false;
    for (int i = 0; i < 3; ++i) st[i] = t->stride(i);
    return true;
}

// (k, v, start, page_table, cache, count, workspace): the error code or None
PyObject *kv4_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 7)) return nullptr;
    const at::Tensor *k = tensor(a[0]), *v = tensor(a[1]);
    long long ks[3], vs[3];
    if (!rows_of_heads(k, ks) || !rows_of_heads(v, vs)) Py_RETURN_NONE;
    const int dev = k->get_device(), code = code_of(k->scalar_type());
    Cache c;
    if (code < 0 || v->scalar_type() != k->scalar_type() || v->get_device() != dev || v->sizes() != k->sizes() ||
        !c.take(dev, k->size(0), a[4], a[3], a[2], a[5], a[6]) || c.heads != k->size(2))
        Py_RETURN_NONE;
    return PyLong_FromLong(unlocked([&] {
        return g_entry.append(k->const_data_ptr(), v->const_data_ptr(), code, ks, vs, c.first, c.second,
                              static_cast<int>(k->size(0)), static_cast<int>(k->size(1)), c.heads, IP_DH, c.table,
                              c.width, c.pages, c.n_pages, c.page, c.ws, c.ws_bytes, stream_of(dev));
    }));
    END_HANDLE_TH_ERRORS
}

// (cache, start, page_table, T, count, dtype, workspace)
PyObject *kv4_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 7)) return nullptr;
    const at::Tensor *cache = tensor(a[0]), *start = tensor(a[1]);
    if (!cache || !start || start->dim() != 1 || !PyLong_CheckExact(a[3]) || !THPDtype_Check(a[5])) Py_RETURN_NONE;
    const at::ScalarType type = reinterpret_cast<THPDtype *>(a[5])->scalar_type;
    const int dev = cache->get_device(), code = code_of(type);
    int over = 0;
    const long T = PyLong_AsLongAndOverflow(a[3], &over);
    Cache c;
    if (code < 0 || over || T < 0 || !fits(T) || !c.take(dev, start->size(0), a[0], a[2], a[1], a[4], a[6]))
        Py_RETURN_NONE;
    const int64_t B = start->size(0), shape[4] = {B, T, c.heads, IP_DH};
    const at::Tensor k = empty(shape, *cache, type), v = empty(shape, *cache, type);
    const int rc = unlocked([&] {
        return g_entry.read(c.pages, c.n_pages, c.page, c.table, c.width, c.first, c.second, static_cast<int>(B),
                            static_cast<int>(T), c.heads, IP_DH, k.data_ptr(), v.data_ptr(), code, c.ws, c.ws_bytes,
                            stream_of(dev));
    });
    return rc == IP_OK ? pair(k, v) : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// (q, lengths, page_table, cache, count, causal, scale, max_len, out, workspace)
PyObject *kv4_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 10)) return nullptr;
    const at::Tensor *q = tensor(a[0]);
    long long qs[3];
    if (!rows_of_heads(q, qs) || !PyBool_Check(a[5]) || (a[6] != Py_None && !PyFloat_CheckExact(a[6])) ||
        (a[7] != Py_None && !PyLong_CheckExact(a[7])))
        Py_RETURN_NONE;
    const int dev = q->get_device(), code = code_of(q->scalar_type());
    Cache c;
    if (code <= 0 || !c.take(dev, q->size(0), a[3], a[2], a[1], a[4], a[9])) Py_RETURN_NONE;
    int over = 0;
    const long max_len = a[7] == Py_None ? static_cast<long>(c.width) * c.page : PyLong_AsLongAndOverflow(a[7], &over);
    if (over || !fits(max_len) || max_len < 0) Py_RETURN_NONE;
    const float scale = a[6] == Py_None ? 0.08838834764831845f : static_cast<float>(PyFloat_AS_DOUBLE(a[6]));
    at::Tensor out;
    if (!output(a[8], q->sizes(), *q, q->scalar_type(), out)) Py_RETURN_NONE;
    const int rc = unlocked([&] {
        return g_entry.attention(q->const_data_ptr(), code, qs, c.first, c.second, a[5] == Py_True ? 1 : 0, scale,
                                 static_cast<int>(q->size(0)), static_cast<int>(q->size(1)),
                                 static_cast<int>(q->size(2)), c.heads, IP_DH, static_cast<int>(max_len), c.table,
                                 c.width, c.pages, c.n_pages, c.page, out.data_ptr(), c.ws, c.ws_bytes, stream_of(dev));
    });
    return rc == IP_OK ? THPVariable_Wrap(out) : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// Addresses of the five entry points, in the order of Entries.
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!arity(n, 5)) return nullptr;
    void *p[5];
    for (int i = 0; i < 5; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_entry = {reinterpret_cast<decltype(g_entry.quantize)>(p[0]), reinterpret_cast<decltype(g_entry.linear)>(p[1]),
               reinterpret_cast<decltype(g_entry.append)>(p[2]), reinterpret_cast<decltype(g_entry.read)>(p[3]),
               reinterpret_cast<decltype(g_entry.attention)>(p[4])};
    Py_RETURN_NONE;
}

template <typename F>
PyMethodDef method(const char *name, F f) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {method("bind", bind), method("quantize_rows", quantize_rows),
                           method("linear_scaled", linear_scaled), method("kv4_append", kv4_append),
                           method("kv4_read", kv4_read), method("kv4_attention", kv4_attention),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "ip_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject *PyInit_ip_torch() { return PyModule_Create(&g_module); }
