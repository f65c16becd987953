// Short forms of the Python calls with run-time scales, on 4-bit rows and on the 4-bit cache, for their usual
// arguments: plain contiguous tensors (or matrices) of the current device, its current stream.
// Each makes the checks of the general form in place, allocates the outputs and calls the C
// entry point; it returns the outputs, the entry point's error code, or None for arguments that
// the general form (Python, over ctypes) has to look at.  A decoder's single-token calls are
// shorter on the GPU than this work takes in Python.
#include <Python.h>

#include <ATen/Context.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <ATen/record_function.h>
#include <c10/core/Storage.h>
#include <c10/core/TensorImpl.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <climits>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "ip_mhsa.h"

namespace {

// The entry points of the library that Python has loaded.
struct Entries {
    decltype(&ip_quantize_rows_i8) quantize;
    decltype(&ip_linear_scaled_i8) linear;
    decltype(&ip_kv4_append) append;
    decltype(&ip_kv4_read) read;
    decltype(&ip_kv4_attention) attention;
    decltype(&ip_quantize_fp4) quantize_fp4;
    decltype(&ip_linear_fp4) linear_fp4;
    decltype(&ip_rmsnorm_i8) norm_i8;
    decltype(&ip_rmsnorm_fp4) norm_fp4;
    decltype(&ip_dequantize_i8) values_i8;
    decltype(&ip_dequantize_fp4) values_fp4;
    decltype(&ip_token_logprobs) logprobs;
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

// Whether anything but the allocator has a part in at::empty: a dispatch mode or a trace, a profiler, or the
// deterministic filling of new memory.
bool watched() {
    const at::Context &context = at::globalContext();
    // autocast lets at::empty pass
    const c10::DispatchKeySet keys = c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set - c10::autocast_dispatch_keyset;
    return !keys.empty() || at::hasCallbacks() ||
           (context.deterministicAlgorithms() && context.deterministicFillUninitializedMemory());
}
// n bytes of the current device and stream.
c10::Storage allocate(size_t n) {
    c10::Allocator *a = c10::cuda::CUDACachingAllocator::get();
    return c10::Storage(c10::Storage::use_byte_size_t(), n, a->allocate(n), a, true);
}
// A tensor over memory of the current device from byte `from` on; strides empty: contiguous.
at::Tensor over(c10::Storage memory, size_t from, at::IntArrayRef shape, at::IntArrayRef strides, at::ScalarType type) {
    at::Tensor t = at::detail::make_tensor<at::TensorImpl>(std::move(memory), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                           c10::scalarTypeToTypeMeta(type));
    at::TensorImpl *impl = t.unsafeGetTensorImpl();
    if (strides.empty()) impl->set_sizes_contiguous(shape);
    else impl->set_sizes_and_strides(shape, strides);
    if (from) impl->set_storage_offset(static_cast<int64_t>(from / c10::elementSize(type)));
    return t;
}
int64_t bytes_of(at::IntArrayRef shape, at::ScalarType type) {
    return c10::multiply_integers(shape) * static_cast<int64_t>(c10::elementSize(type));
}

// A new tensor on the current device, which is like's: what at::empty makes, and by it where anything watches; by itself
// 1.0 to 1.3 us less of a Grace core.  strides empty: contiguous; n: the bytes.
at::Tensor empty(at::IntArrayRef shape, at::IntArrayRef strides, const at::Tensor &like, at::ScalarType type, int64_t n) {
    if (!watched()) return over(allocate(static_cast<size_t>(n)), 0, shape, strides, type);
    const at::TensorOptions options = like.options().dtype(type).requires_grad(false);
    at::Tensor t = strides.empty() ? at::empty(shape, options) : at::empty_strided(shape, strides, options);
    // memory of the device: under some dispatch modes a tensor has none, or another's
    TORCH_CHECK(n == 0 || (t.is_cuda() && t.data_ptr() != nullptr), "no memory of the device for an output");
    return t;
}
at::Tensor empty(at::IntArrayRef shape, const at::Tensor &like, at::ScalarType type) {
    return empty(shape, {}, like, type, bytes_of(shape, type));
}

// A call's new outputs, taken piece by piece; like: an input, whose device is the current one.  Outputs of up to
// TOGETHER bytes in all share one allocation, which is what they cost the host most of (a call with four of
// them 4.0 us of a Grace core, 5.1 one by one); larger ones have their own, so that none keeps more than this of
// the others' memory alive.
class Memory {
public:
    static constexpr size_t TOGETHER = 1 << 20;
    // what a piece of n bytes takes
    static size_t piece(int64_t n) { return (static_cast<size_t>(n) + 127) & ~static_cast<size_t>(127); }

    Memory(size_t bytes, const at::Tensor &like) : like_(like), shared_(bytes <= TOGETHER) {
        if (!shared_) return;
        if (!watched()) {
            memory_ = allocate(bytes);
            return;
        }
        memory_ = empty({static_cast<int64_t>(bytes)}, like, at::kByte).storage();
    }
    // strides empty: contiguous; n: the bytes
    at::Tensor take(at::IntArrayRef shape, at::IntArrayRef strides, at::ScalarType type, int64_t n) {
        if (!shared_) return empty(shape, strides, like_, type, n);
        const size_t from = used_;
        used_ += piece(n);
        return over(memory_, from, shape, strides, type);
    }
    at::Tensor take(at::IntArrayRef shape, at::ScalarType type) { return take(shape, {}, type, bytes_of(shape, type)); }

private:
    const at::Tensor &like_;
    bool shared_;
    c10::Storage memory_;
    size_t used_ = 0;
};

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

// Rows of n elements of one byte each, `lead` of them, on multiples of 16 bytes.
struct ByteShape {
    c10::SmallVector<int64_t, 6> shape, strides;
    int64_t ld, bytes;

    ByteShape(at::IntArrayRef lead, int64_t n) : shape(lead.begin(), lead.end()), ld((n + 15) / 16 * 16) {
        shape.push_back(n);
        bytes = c10::multiply_integers(lead) * ld;
        if (ld == n) return;
        strides.resize(shape.size(), 1);
        int64_t step = ld;
        for (size_t i = shape.size() - 1; i-- > 0; step *= shape[i] > 1 ? shape[i] : 1) strides[i] = step;
    }
};

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
        const ByteShape rows(x->sizes().slice(0, x->dim() - 1), d);
        q = empty(rows.shape, rows.strides, *x, at::kChar, rows.bytes);
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

// Tensors as a tuple, None for those that are not there.
PyObject *tuple(std::initializer_list<const at::Tensor *> list) {
    PyObject *r = PyTuple_New(static_cast<Py_ssize_t>(list.size()));
    if (!r) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor *t : list) {
        PyObject *o = Py_None;
        if (t) o = THPVariable_Wrap(*t);
        else Py_INCREF(o);
        if (!o) {
            Py_DECREF(r);
            return nullptr;
        }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}

// Contiguous rows of real values on the current device.
struct Rows {
    const at::Tensor *x;
    int dev, code;
    int64_t d, rows;

    bool take(PyObject *o) {
        x = tensor(o);
        if (!x || x->dim() < 1 || !x->is_contiguous()) return false;
        dev = x->get_device();
        code = code_of(x->scalar_type());
        d = x->size(-1);
        if (code < 0 || d < 1 || !fits(d) || dev != c10::cuda::current_device()) return false;
        rows = x->numel() / d;
        return true;
    }
    at::IntArrayRef lead() const { return x->sizes().slice(0, x->dim() - 1); }
    std::array<int64_t, 3> blocks() const { return {(rows + 127) / 128, (d + 63) / 64, 512}; }
};

// (x, q, blocks, scale), the last three None
PyObject *quantize_fp4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 4)) return nullptr;
    Rows r;
    if (a[1] != Py_None || a[2] != Py_None || a[3] != Py_None || !r.take(a[0])) Py_RETURN_NONE;
    const ByteShape codes(r.lead(), (r.d + 1) / 2);
    const int64_t block_bytes = bytes_of(r.blocks(), at::kByte), ld = codes.ld;
    Memory mem(Memory::piece(codes.bytes) + Memory::piece(block_bytes) + Memory::piece(4 * r.rows), *r.x);
    const at::Tensor q = mem.take(codes.shape, codes.strides, at::kByte, codes.bytes), blocks = mem.take(r.blocks(), at::kByte),
                     scale = mem.take(r.lead(), at::kFloat);
    const int rc = unlocked([&] {
        return g_entry.quantize_fp4(r.x->const_data_ptr(), r.code, r.rows, static_cast<int>(r.d), r.d,
                                    static_cast<uint8_t *>(q.data_ptr()), ld, static_cast<uint8_t *>(blocks.data_ptr()),
                                    static_cast<float *>(scale.data_ptr()), stream_of(r.dev));
    });
    return rc == IP_OK ? tuple({&q, &blocks, &scale}) : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// (x, weight, residual, eps, out, q, blocks, scale), the last three None (i8: without blocks)
PyObject *norm(PyObject *const *a, Py_ssize_t n, bool fp4) {
    HANDLE_TH_ERRORS
    if (!arity(n, fp4 ? 8 : 7)) return nullptr;
    Rows r;
    for (Py_ssize_t i = 5; i < n; ++i)
        if (a[i] != Py_None) Py_RETURN_NONE;
    if (!PyFloat_CheckExact(a[3]) || !r.take(a[0])) Py_RETURN_NONE;
    const at::ScalarType type = r.x->scalar_type();
    const at::Tensor *w = tensor(a[1]), *res = nullptr;
    if (!vector(w, type, r.d, r.dev)) Py_RETURN_NONE;
    at::Tensor sum;
    const bool new_sum = a[2] != Py_None && a[4] == Py_None;
    if (a[2] != Py_None) {
        res = tensor(a[2]);
        if (!contiguous(res, type, r.dev) || res->sizes() != r.x->sizes() ||
            (!new_sum && !output(a[4], r.x->sizes(), *r.x, type, sum)))
            Py_RETURN_NONE;
    } else if (a[4] != Py_None) {
        Py_RETURN_NONE;
    }
    const ByteShape codes(r.lead(), fp4 ? (r.d + 1) / 2 : r.d);
    const int64_t block_bytes = fp4 ? bytes_of(r.blocks(), at::kByte) : 0, ld = codes.ld;
    const int64_t sum_bytes = new_sum ? bytes_of(r.x->sizes(), type) : 0;
    Memory mem(Memory::piece(codes.bytes) + Memory::piece(block_bytes) + Memory::piece(4 * r.rows) + Memory::piece(sum_bytes), *r.x);
    const at::Tensor q = mem.take(codes.shape, codes.strides, fp4 ? at::kByte : at::kChar, codes.bytes);
    const at::Tensor scale = mem.take(r.lead(), at::kFloat);
    at::Tensor blocks;
    if (fp4) blocks = mem.take(r.blocks(), at::kByte);
    if (new_sum) sum = mem.take(r.x->sizes(), type);
    const float eps = static_cast<float>(PyFloat_AS_DOUBLE(a[3]));
    const void *pr = res ? res->const_data_ptr() : nullptr;
    void *ps = res ? sum.data_ptr() : nullptr;
    const int d = static_cast<int>(r.d);
    const int rc = unlocked([&] {
        return fp4 ? g_entry.norm_fp4(r.x->const_data_ptr(), d, pr, d, w->const_data_ptr(), eps, r.code, r.rows, d, ps, d,
                                      static_cast<uint8_t *>(q.data_ptr()), ld, static_cast<uint8_t *>(blocks.data_ptr()),
                                      static_cast<float *>(scale.data_ptr()), stream_of(r.dev))
                   : g_entry.norm_i8(r.x->const_data_ptr(), d, pr, d, w->const_data_ptr(), eps, r.code, r.rows, d, ps, d,
                                     static_cast<int8_t *>(q.data_ptr()), ld, static_cast<float *>(scale.data_ptr()),
                                     stream_of(r.dev));
    });
    if (rc != IP_OK) return PyLong_FromLong(rc);
    const at::Tensor *total = res ? &sum : nullptr;
    return fp4 ? tuple({&q, &blocks, &scale, total}) : tuple({&q, &scale, total});
    END_HANDLE_TH_ERRORS
}
PyObject *rmsnorm_i8(PyObject *, PyObject *const *a, Py_ssize_t n) { return norm(a, n, false); }
PyObject *rmsnorm_fp4(PyObject *, PyObject *const *a, Py_ssize_t n) { return norm(a, n, true); }

// The type that a call writes: `dtype`, else out's, else bfloat16; false for what the general form has to look at.
bool type_of(PyObject *dtype, PyObject *out, at::ScalarType &type) {
    type = at::kBFloat16;
    if (THPDtype_Check(dtype)) type = reinterpret_cast<THPDtype *>(dtype)->scalar_type;
    else if (dtype != Py_None) return false;
    else if (THPVariable_CheckExact(out)) type = THPVariable_Unpack(out).scalar_type();
    return code_of(type) >= 0;
}

// Stride of rows whose leading axes are walked with one, 0 for what the general form has to look at.
int64_t rows_stride(const at::Tensor &t) {
    if (t.stride(-1) != 1 && t.size(-1) != 1) return 0;
    if (t.numel() <= t.size(-1)) return (t.size(-1) + 15) / 16 * 16;      // one row or none: any stride does
    int64_t ld = 0, rows = 1;
    for (int64_t i = t.dim() - 2; i >= 0; --i) {
        if (t.size(i) != 1) {
            if (ld == 0) ld = t.stride(i);
            else if (t.stride(i) != ld * rows) return 0;
        }
        rows *= t.size(i);
    }
    return ld;
}

// Rows of bytes with a scale each, and for 4-bit rows (d elements, -1: two a byte) their blocks.
struct ByteRows {
    const at::Tensor *q, *scale, *blocks;
    int64_t rows, d, ld;

    bool take(PyObject *oq, PyObject *oscale, PyObject *oblocks, int64_t want, int dev) {
        q = tensor(oq), scale = tensor(oscale), blocks = oblocks ? tensor(oblocks) : nullptr;
        if (!q || q->dim() < 1 || q->scalar_type() != (oblocks ? at::kByte : at::kChar) || q->get_device() != dev ||
            !contiguous(scale, at::kFloat, dev))
            return false;
        const int64_t n = q->size(-1);
        if (n < 1 || n > INT_MAX / 2 || scale->sizes() != lead()) return false;
        d = oblocks ? (want < 0 ? 2 * n : want) : n;
        rows = q->numel() / n;
        ld = rows_stride(*q);
        if (ld < n) return false;
        if (!oblocks) return true;
        return (d + 1) / 2 == n && contiguous(blocks, at::kByte, dev) && blocks->dim() == 3 &&
               blocks->size(0) == (rows + 127) / 128 && blocks->size(1) == (d + 63) / 64 && blocks->size(2) == 512;
    }
    at::IntArrayRef lead() const { return q->sizes().slice(0, q->dim() - 1); }
    const uint8_t *codes() const { return static_cast<const uint8_t *>(q->const_data_ptr()); }
    const uint8_t *scales() const { return static_cast<const uint8_t *>(blocks->const_data_ptr()); }
    const float *factors() const { return static_cast<const float *>(scale->const_data_ptr()); }
};

PyObject *values(PyObject *oq, PyObject *oscale, PyObject *oblocks, int64_t d, PyObject *dtype, PyObject *o) {
    const at::Tensor *q = tensor(oq);
    ByteRows r;
    at::ScalarType type;
    if (!q || !type_of(dtype, o, type)) Py_RETURN_NONE;
    const int dev = q->get_device();
    if (dev != c10::cuda::current_device() || !r.take(oq, oscale, oblocks, d, dev)) Py_RETURN_NONE;
    c10::SmallVector<int64_t, 6> shape(r.lead().begin(), r.lead().end());
    shape.push_back(r.d);
    at::Tensor out;
    if (!output(o, shape, *r.q, type, out)) Py_RETURN_NONE;
    const int rc = unlocked([&] {
        return oblocks ? g_entry.values_fp4(r.codes(), r.ld, r.scales(), r.factors(), r.rows, static_cast<int>(r.d),
                                            out.data_ptr(), r.d, code_of(type), stream_of(dev))
                       : g_entry.values_i8(reinterpret_cast<const int8_t *>(r.codes()), r.ld, r.factors(), r.rows,
                                           static_cast<int>(r.d), out.data_ptr(), r.d, code_of(type), stream_of(dev));
    });
    return rc == IP_OK ? THPVariable_Wrap(out) : PyLong_FromLong(rc);
}
// (q, scale, dtype, out)
PyObject *dequantize_i8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 4)) return nullptr;
    return values(a[0], a[1], nullptr, -1, a[2], a[3]);
    END_HANDLE_TH_ERRORS
}
// (q, blocks, scale, d, dtype, out)
PyObject *dequantize_fp4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 6)) return nullptr;
    int64_t d = -1;
    if (a[3] != Py_None) {
        int over = 0;
        if (!PyLong_CheckExact(a[3])) Py_RETURN_NONE;
        d = PyLong_AsLongAndOverflow(a[3], &over);
        if (over || d < 1 || !fits(d)) Py_RETURN_NONE;
    }
    return values(a[0], a[2], a[1], d, a[4], a[5]);
    END_HANDLE_TH_ERRORS
}

// (x, x_blocks, sx, w, w_blocks, sw, bias, act, dtype, out, workspace)
PyObject *linear_fp4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 11)) return nullptr;
    const at::Tensor *ws = tensor(a[10]);
    at::ScalarType type;
    if (!ws || !PyLong_CheckExact(a[7]) || !type_of(a[8], a[9], type)) Py_RETURN_NONE;
    const int dev = ws->get_device();
    ByteRows x, w;
    if (dev != c10::cuda::current_device() || !contiguous(ws, at::kByte, dev) || !x.take(a[0], a[2], a[1], -1, dev) ||
        !w.take(a[3], a[5], a[4], -1, dev) || w.q->dim() != 2 || w.d != x.d || (x.ld | w.ld) % 16 != 0 || w.rows < 1 ||
        !fits(w.rows))
        Py_RETURN_NONE;
    int over = 0;
    const long act = PyLong_AsLongAndOverflow(a[7], &over);
    const void *bias;
    if (over || act < 0 || act > INT_MAX || !maybe_vector(a[6], at::kFloat, w.rows, dev, bias)) Py_RETURN_NONE;
    c10::SmallVector<int64_t, 6> shape(x.lead().begin(), x.lead().end());
    shape.push_back(w.rows);
    at::Tensor out;
    if (!output(a[9], shape, *x.q, type, out)) Py_RETURN_NONE;
    const int rc = unlocked([&] {
        return g_entry.linear_fp4(x.codes(), x.ld, x.scales(), x.factors(), w.codes(), w.ld, w.scales(), w.factors(),
                                  static_cast<const float *>(bias), static_cast<int>(act), x.rows, static_cast<int>(x.d),
                                  static_cast<int>(w.rows), out.data_ptr(), w.rows, code_of(type), ws->data_ptr(),
                                  static_cast<size_t>(ws->numel()), stream_of(dev));
    });
    return rc == IP_OK ? THPVariable_Wrap(out) : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// (logits, tokens, top, scale, workspace)
PyObject *token_logprobs(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arity(n, 5)) return nullptr;
    const at::Tensor *x = tensor(a[0]), *tok = nullptr, *ws = tensor(a[4]);
    if (!x || !ws || x->dim() < 1 || !PyLong_CheckExact(a[2]) || !PyFloat_CheckExact(a[3])) Py_RETURN_NONE;
    const int dev = x->get_device(), code = code_of(x->scalar_type());
    const int64_t V = x->size(-1), ld = V < 1 ? 0 : row_stride(*x);
    int over = 0;
    const long top = PyLong_AsLongAndOverflow(a[2], &over);
    if (code < 0 || dev != c10::cuda::current_device() || V < 1 || !fits(V) || ld < V || over || top < 0 ||
        top > IP_LOGPROBS_MAX_TOP || !contiguous(ws, at::kByte, dev))
        Py_RETURN_NONE;
    const at::IntArrayRef lead = x->sizes().slice(0, x->dim() - 1);
    bool wide = false;
    if (a[1] != Py_None) {
        tok = tensor(a[1]);
        if (!tok || !tok->is_contiguous() || tok->get_device() != dev || tok->sizes() != lead) Py_RETURN_NONE;
        wide = tok->scalar_type() == at::kLong;
        if (!wide && tok->scalar_type() != at::kInt) Py_RETURN_NONE;
    }
    const int64_t rows = x->numel() / V;
    Memory mem(2 * Memory::piece(4 * rows) + 2 * Memory::piece(4 * rows * top), *x);
    at::Tensor lp, ent = mem.take(lead, at::kFloat), tlp, ttok;
    if (tok) lp = mem.take(lead, at::kFloat);
    if (top > 0) {
        c10::SmallVector<int64_t, 6> shape(lead.begin(), lead.end());
        shape.push_back(top);
        tlp = mem.take(shape, at::kFloat);
        ttok = mem.take(shape, at::kInt);
    }
    const float scale = static_cast<float>(PyFloat_AS_DOUBLE(a[3]));
    auto data = [](const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
    const int rc = unlocked([&] {
        return g_entry.logprobs(x->const_data_ptr(), code, rows, static_cast<int>(V), ld,
                                tok ? tok->const_data_ptr() : nullptr, wide ? 1 : 0, scale, static_cast<int>(top),
                                static_cast<float *>(data(lp)), static_cast<float *>(data(ent)),
                                static_cast<float *>(data(tlp)), static_cast<int32_t *>(data(ttok)), ws->data_ptr(),
                                static_cast<size_t>(ws->numel()), stream_of(dev));
    });
    if (rc != IP_OK) return PyLong_FromLong(rc);
    return tuple({tok ? &lp : nullptr, &ent, top > 0 ? &tlp : nullptr, top > 0 ? &ttok : nullptr});
    END_HANDLE_TH_ERRORS
}

// Addresses of the entry points, in the order of Entries.
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    constexpr int N = 12;
    if (!arity(n, N)) return nullptr;
    void *p[N];
    for (int i = 0; i < N; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    int i = 0;
    auto take = [&](auto &f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(p[i++]); };
    take(g_entry.quantize);
    take(g_entry.linear);
    take(g_entry.append);
    take(g_entry.read);
    take(g_entry.attention);
    take(g_entry.quantize_fp4);
    take(g_entry.linear_fp4);
    take(g_entry.norm_i8);
    take(g_entry.norm_fp4);
    take(g_entry.values_i8);
    take(g_entry.values_fp4);
    take(g_entry.logprobs);
    Py_RETURN_NONE;
}

template <typename F>
PyMethodDef method(const char *name, F f) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {method("bind", bind), method("quantize_rows", quantize_rows),
                           method("linear_scaled", linear_scaled), method("kv4_append", kv4_append),
                           method("kv4_read", kv4_read), method("kv4_attention", kv4_attention),
                           method("quantize_fp4", quantize_fp4), method("linear_fp4", linear_fp4),
                           method("rmsnorm_i8", rmsnorm_i8), method("rmsnorm_fp4", rmsnorm_fp4),
                           method("dequantize_i8", dequantize_i8), method("dequantize_fp4", dequantize_fp4),
                           method("token_logprobs", token_logprobs),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "ip_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject *PyInit_ip_torch() { return PyModule_Create(&g_module); }
