// The hot entry points of include/fq.h for torch tensors, as a CPython module: shape and type checks, output and
// workspace from torch's caching allocator, torch's current stream, one call into the library.  Marshalling only, like
// fq.py, which wraps these functions; it is native because an eager call on a short batch is bound by it: the kernels of
// a 64-token projection take 7 us, and a call marshalled through ctypes and torch.empty took 19.4 us of host time
// (at most 8.5 us here, its two launches included; M = 64, K = N = 1024).
//
// Every function returns its result, or the fq_status (an int) of a call that was refused.  All that is read from Python
// objects is read first; then the interpreter lock is given up for the allocations and the call into the library, as ctypes
// and torch do: a launch waits while its stream's queue is full, and other Python threads -- a function that the stream itself
// calls on the host among them, for which that queue may be waiting -- have to run meanwhile.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "fq.h"

namespace {

struct Refused {};          // a Python exception is set

// The interpreter lock given up for a scope, exceptions included.
class Unlocked {
public:
    Unlocked() : state_(PyEval_SaveThread()) {}
    ~Unlocked() { PyEval_RestoreThread(state_); }
    Unlocked(const Unlocked&) = delete;
    Unlocked& operator=(const Unlocked&) = delete;

private:
    PyThreadState* state_;
};

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a torch.Tensor, got %s", Py_TYPE(o)->tp_name);
        throw Refused();
    }
    return THPVariable_Unpack(o);
}
const at::Tensor& rowmajor(PyObject* o) {
    const at::Tensor& t = tensor(o);
    if (t.dim() != 2 || t.stride(1) != 1) {
        PyErr_SetString(PyExc_ValueError, "expected a 2-D tensor with unit inner stride");
        throw Refused();
    }
    return t;
}
long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
}
void* address(PyObject* o) { return reinterpret_cast<void*>(static_cast<uintptr_t>(integer(o))); }
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return static_cast<float>(v);
}
fq_dtype dtype_of(at::ScalarType t) {
    if (t == at::kFloat) return FQ_F32;
    if (t == at::kBFloat16) return FQ_BF16;
    PyErr_Format(PyExc_TypeError, "unsupported dtype %s", at::toString(t));
    throw Refused();
}
void arguments(Py_ssize_t got, Py_ssize_t wanted) {
    if (got != wanted) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", wanted, got);
        throw Refused();
    }
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }
bool none(PyObject* o) { return o == Py_None; }
PyObject* status(fq_status s) { return PyLong_FromLong(s); }

// (on a GPU straight from the allocator: at::empty's way through the dispatcher costs as much again)
at::Tensor fresh(at::IntArrayRef size, at::ScalarType t, const at::Tensor& like) {
    if (like.is_cuda()) return at::Tensor(at::detail::empty_cuda(size, t, like.device(), std::nullopt));
    return at::empty(size, at::TensorOptions().dtype(t).device(like.device()));
}

// An output: the caller's tensor (its own dtype decides) or, made by make(), a new one of `dtype` on x's device.
struct Output {
    at::Tensor t;
    at::ScalarType type;
    fq_dtype dt;
    Output(PyObject* given, PyObject* dtype) {
        if (!none(given)) {
            t = tensor(given);
            type = t.scalar_type();
        } else if (THPDtype_Check(dtype)) {
            type = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
        } else {
            PyErr_SetString(PyExc_TypeError, "out_dtype has to be a torch.dtype");
            throw Refused();
        }
        dt = dtype_of(type);
    }
    Output(PyObject* given, at::ScalarType otherwise) : type(otherwise), dt(FQ_F32) {
        if (!none(given)) t = tensor(given);
    }
    void make(at::IntArrayRef size, const at::Tensor& like) {
        if (!t.defined()) t = fresh(size, type, like);
    }
};

// The caller's workspace, or one from torch's allocator for the length of the call: it is handed back when the kernels
// are enqueued, and the allocator gives it to later work of this stream only -- what a torch.empty that goes out of
// scope does.
struct Workspace {
    void* p = nullptr;
    size_t bytes = 0;
    at::Tensor own;
    explicit Workspace(PyObject* given) {
        if (none(given)) return;
        const at::Tensor& t = tensor(given);
        p = t.data_ptr();
        bytes = static_cast<size_t>(t.numel());
        given_ = true;
    }
    template <typename Need>
    void make(Need need, const at::Tensor& like) {
        if (given_) return;
        bytes = need();
        own = fresh({static_cast<int64_t>(bytes)}, at::kByte, like);
        p = own.data_ptr();
    }

private:
    bool given_ = false;
};

PyObject* pair(at::Tensor&& a, at::Tensor&& b) {
    PyObject* r = PyTuple_New(2);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(std::move(a)));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(std::move(b)));
    return r;
}

template <typename F>
PyObject* guarded(F f) {
    HANDLE_TH_ERRORS
    try {
        return f();
    } catch (const Refused&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// The arguments that the one-call entry points share: (x, handle, K, N, handle_bits, ., clip_ratio, out_dtype, y, workspace)
template <typename F>
PyObject* one_call(PyObject* const* a, Py_ssize_t n, F run) {
    return guarded([&]() -> PyObject* {
        arguments(n, 10);
        const at::Tensor& x = rowmajor(a[0]);
        const fq_weights* W = static_cast<const fq_weights*>(address(a[1]));
        const int64_t K = integer(a[2]), N = integer(a[3]), M = x.size(0);
        const int handle_bits = static_cast<int>(integer(a[4]));
        const long long which = integer(a[5]);
        const float clip = real(a[6]);
        const fq_dtype xt = dtype_of(x.scalar_type());
        const void* xp = x.data_ptr();
        const int64_t ldx = x.stride(0);
        Output y(a[8], a[7]);
        Workspace ws(a[9]);
        fq_status s;
        {
            const Unlocked nogil;
            y.make({M, N}, x);
            ws.make([&] { return fq_workspace_bytes(M, K, N, handle_bits); }, x);
            s = run(which, xp, xt, M, ldx, W, clip, y.t.data_ptr(), y.dt, y.t.stride(0), ws.p, ws.bytes);
        }
        return s == FQ_OK ? THPVariable_Wrap(std::move(y.t)) : status(s);
    });
}

// linear(x, handle, K, N, handle_bits, bits, clip_ratio, out_dtype, y, workspace): fq_linear_w4a4 / _w8a8 by `bits`
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return one_call(a, n, [](long long bits, const void* x, fq_dtype xt, int64_t M, int64_t ldx, const fq_weights* W, float clip,
                             void* y, fq_dtype yt, int64_t ldy, void* ws, size_t ws_bytes) {
        return (bits == 4 ? fq_linear_w4a4 : fq_linear_w8a8)(x, xt, M, ldx, W, clip, y, yt, ldy, ws, ws_bytes, stream());
    });
}

// linear_gated(x, handle, K, N, handle_bits, act, clip_ratio, out_dtype, y, workspace): fq_linear_gated.  (`act` is the
// caller's: whatever is neither function is refused as the library refuses it, ahead of its narrowing to the enumeration.)
PyObject* linear_gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return one_call(a, n, [](long long act, const void* x, fq_dtype xt, int64_t M, int64_t ldx, const fq_weights* W, float clip,
                             void* y, fq_dtype yt, int64_t ldy, void* ws, size_t ws_bytes) {
        if (act != FQ_GATE_SILU && act != FQ_GATE_GELU_TANH) return FQ_ERR_INVALID_ARG;
        return fq_linear_gated(x, xt, M, ldx, static_cast<fq_gate_act>(act), W, clip, y, yt, ldy, ws, ws_bytes, stream());
    });
}

// gemm(codes, delta, handle, K, N, handle_bits, bits, out_dtype, y, workspace): fq_gemm_w4a4 / fq_gemm_w8a8 by `bits`
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 10);
        const at::Tensor &codes = tensor(a[0]), &delta = tensor(a[1]);
        const fq_weights* W = static_cast<const fq_weights*>(address(a[2]));
        const int64_t K = integer(a[3]), N = integer(a[4]), M = codes.size(0);
        const int handle_bits = static_cast<int>(integer(a[5])), bits = static_cast<int>(integer(a[6]));
        const void* cp = codes.data_ptr();
        const float* dp = static_cast<const float*>(delta.data_ptr());
        Output y(a[8], a[7]);
        Workspace ws(a[9]);
        fq_status s;
        {
            const Unlocked nogil;
            y.make({M, N}, codes);
            ws.make([&] { return fq_workspace_bytes(M, K, N, handle_bits); }, codes);
            s = (bits == 4 ? fq_gemm_w4a4 : fq_gemm_w8a8)(cp, dp, M, W, y.t.data_ptr(), y.dt, y.t.stride(0), ws.p, ws.bytes, stream());
        }
        return s == FQ_OK ? THPVariable_Wrap(std::move(y.t)) : status(s);
    });
}

// quantize_act(x, multiplier address, block, bits, clip_ratio, codes, delta, fold_after) -> (codes, delta)
PyObject* quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 8);
        const at::Tensor& x = rowmajor(a[0]);
        const float* g = static_cast<const float*>(address(a[1]));
        const int64_t M = x.size(0), K = x.size(1);
        const int block = static_cast<int>(integer(a[2])), bits = static_cast<int>(integer(a[3]));
        const float clip = real(a[4]);
        const fq_dtype xt = dtype_of(x.scalar_type());
        const bool after = integer(a[7]) != 0;
        const void* xp = x.data_ptr();
        const int64_t ldx = x.stride(0);
        Output codes(a[5], at::kByte), delta(a[6], at::kFloat);
        fq_status s;
        {
            const Unlocked nogil;
            codes.make({M, K * bits / 8}, x);
            delta.make({M}, x);
            s = (after ? fq_quantize_act_after : fq_quantize_act)(xp, xt, M, K, ldx, g, block, bits, clip, codes.t.data_ptr(),
                                                                  static_cast<float*>(delta.t.data_ptr()), stream());
        }
        return s == FQ_OK ? pair(std::move(codes.t), std::move(delta.t)) : status(s);
    });
}

// quantize_act_composite(x, multiplier address, perm, blocks, bits, clip_ratio, codes, delta, workspace) -> (codes, delta)
PyObject* quantize_act_composite(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 9);
        const at::Tensor& x = rowmajor(a[0]);
        const float* g = static_cast<const float*>(address(a[1]));
        const at::Tensor &perm = tensor(a[2]), &blocks = tensor(a[3]);
        if (perm.scalar_type() != at::kInt || blocks.scalar_type() != at::kFloat || !blocks.is_contiguous() || blocks.dim() != 3) {
            PyErr_SetString(PyExc_AssertionError, "perm has to be int32, blocks contiguous float32 [K/block, block, block]");
            throw Refused();
        }
        const int64_t M = x.size(0), K = x.size(1);
        const int bits = static_cast<int>(integer(a[4]));
        const float clip = real(a[5]);
        const fq_dtype xt = dtype_of(x.scalar_type());
        const void* xp = x.data_ptr();
        const int64_t ldx = x.stride(0);
        const int32_t* pp = perm.data_ptr<int32_t>();
        const float* bp = blocks.data_ptr<float>();
        const int block = static_cast<int>(blocks.size(1));
        Output codes(a[6], at::kByte), delta(a[7], at::kFloat);
        Workspace ws(a[8]);
        fq_status s;
        {
            const Unlocked nogil;
            codes.make({M, K * bits / 8}, x);
            delta.make({M}, x);
            ws.make([&] { return static_cast<size_t>(M * K > 4 ? 4 * M * K : 16); }, x);
            s = fq_quantize_act_composite(xp, xt, M, K, ldx, g, pp, bp, block, bits, clip, codes.t.data_ptr(),
                                          static_cast<float*>(delta.t.data_ptr()), ws.p, ws.bytes, stream());
        }
        return s == FQ_OK ? pair(std::move(codes.t), std::move(delta.t)) : status(s);
    });
}

// linear_w4a16(x, handle, N, out_dtype, y)
PyObject* linear_w4a16(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 5);
        const at::Tensor& x = rowmajor(a[0]);
        const fq_weights* W = static_cast<const fq_weights*>(address(a[1]));
        const int64_t N = integer(a[2]), M = x.size(0);
        const fq_dtype xt = dtype_of(x.scalar_type());
        const void* xp = x.data_ptr();
        const int64_t ldx = x.stride(0);
        Output y(a[4], a[3]);
        fq_status s;
        {
            const Unlocked nogil;
            y.make({M, N}, x);
            s = fq_linear_w4a16(xp, xt, M, ldx, W, y.t.data_ptr(), y.dt, y.t.stride(0), stream());
        }
        return s == FQ_OK ? THPVariable_Wrap(std::move(y.t)) : status(s);
    });
}

// ---- the operators between a layer's projections ----
// A tensor that the kernels of the current device and stream read or write.
const at::Tensor& on_device(const at::Tensor& t, const char* what) {
    if (!t.is_cuda() || t.device().index() != c10::cuda::current_device()) {
        PyErr_Format(PyExc_ValueError, "%s has to be on the current CUDA device", what);
        throw Refused();
    }
    return t;
}
const at::Tensor& vector_of(PyObject* o, at::ScalarType type, int64_t size, const char* what) {
    const at::Tensor& t = on_device(tensor(o), what);
    if (t.scalar_type() != type || t.dim() != 1 || !t.is_contiguous() || t.size(0) != size) {
        PyErr_Format(PyExc_ValueError, "%s has to be a contiguous %s tensor of %lld elements", what, at::toString(type), (long long)size);
        throw Refused();
    }
    return t;
}
template <typename T>
T* data_or_null(PyObject* o, at::ScalarType type, int64_t size, const char* what) {
    return none(o) ? nullptr : static_cast<T*>(vector_of(o, type, size, what).data_ptr());
}
const at::Tensor& rows_of(PyObject* o, int64_t width, const char* what) {
    const at::Tensor& t = on_device(rowmajor(o), what);
    if (t.size(1) != width) {
        PyErr_Format(PyExc_ValueError, "%s has to have %lld columns, got %lld", what, (long long)width, (long long)t.size(1));
        throw Refused();
    }
    return t;
}
// (the stride between the rows of a matrix of one row is whatever a view left there)
int64_t pitch(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : (t.size(1) + 7) / 8 * 8; }

struct RowsOut {
    at::Tensor t;
    RowsOut(PyObject* given, int64_t rows, int64_t width, at::ScalarType type, const char* what) {
        if (none(given)) return;
        t = rows_of(given, width, what);
        if (t.size(0) != rows || t.scalar_type() != type) {
            PyErr_Format(PyExc_ValueError, "%s has to have %lld rows of %s", what, (long long)rows, at::toString(type));
            throw Refused();
        }
    }
    void make(int64_t rows, int64_t width, at::ScalarType type, const at::Tensor& like) {
        if (!t.defined()) t = fresh({rows, width}, type, like);
    }
};

// qk_norm_rope(qkv, q_heads, k_heads, head_dim, positions, frequencies, q_gain, k_gain, eps, layout, amplitude, out_dtype, q, k) -> (q, k)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 14);
        const at::Tensor& x = on_device(rowmajor(a[0]), "qkv");
        const int64_t q_heads = integer(a[1]), k_heads = integer(a[2]), D = integer(a[3]), M = x.size(0);
        if (q_heads < 0 || k_heads < 0 || D < 1 || q_heads > 32767 || k_heads > 32767 || D > 256) return status(q_heads < 0 || k_heads < 0 || D < 1 ? FQ_ERR_INVALID_ARG : FQ_ERR_UNSUPPORTED);
        if (x.size(1) < (q_heads + k_heads) * D) return status(FQ_ERR_INVALID_ARG);
        const int32_t* positions = static_cast<int32_t*>(vector_of(a[4], at::kInt, M, "positions").data_ptr());
        const at::Tensor& freq = tensor(a[5]);
        const int64_t half = freq.dim() == 1 ? freq.size(0) : 0;
        const double* frequencies = static_cast<double*>(vector_of(a[5], at::kDouble, half, "frequencies").data_ptr());
        const float* q_gain = data_or_null<float>(a[6], at::kFloat, D, "q_gain");
        const float* k_gain = data_or_null<float>(a[7], at::kFloat, D, "k_gain");
        const float eps = real(a[8]), amplitude = real(a[10]);
        const long long layout = integer(a[9]);
        if (layout != FQ_ROPE_HALF && layout != FQ_ROPE_INTERLEAVED) return status(FQ_ERR_INVALID_ARG);
        const fq_dtype xt = dtype_of(x.scalar_type());
        at::ScalarType type = x.scalar_type();
        if (!none(a[11])) {
            if (!THPDtype_Check(a[11])) {
                PyErr_SetString(PyExc_TypeError, "out_dtype has to be a torch.dtype");
                throw Refused();
            }
            type = reinterpret_cast<THPDtype*>(a[11])->scalar_type;
        } else if (!none(a[12])) {
            type = tensor(a[12]).scalar_type();
        }
        const fq_dtype yt = dtype_of(type);
        RowsOut q(a[12], M, q_heads * D, type, "q"), k(a[13], M, k_heads * D, type, "k");
        fq_status s;
        {
            const Unlocked nogil;
            q.make(M, q_heads * D, type, x);
            k.make(M, k_heads * D, type, x);
            s = fq_qk_norm_rope(x.data_ptr(), xt, M, pitch(x), (int)q_heads, (int)k_heads, (int)D, q_gain, k_gain, eps, positions, frequencies,
                                (int)(2 * half), static_cast<fq_rope_layout>(layout), amplitude, q.t.data_ptr(), pitch(q.t), k.t.data_ptr(), pitch(k.t),
                                yt, stream());
        }
        return s == FQ_OK ? pair(std::move(q.t), std::move(k.t)) : status(s);
    });
}

// The tensors of a cache, (k, v, k_scale, v_scale), checked when the Python object was made.
fq_kv8_cache cache_of(PyObject* const* a) {
    const at::Tensor &k = on_device(tensor(a[0]), "the cache"), &v = on_device(tensor(a[1]), "the cache");
    const at::Tensor &ks = on_device(tensor(a[2]), "the cache"), &vs = on_device(tensor(a[3]), "the cache");
    fq_kv8_cache c = {};
    c.k = static_cast<int8_t*>(k.data_ptr());
    c.v = static_cast<int8_t*>(v.data_ptr());
    c.k_scale = static_cast<float*>(ks.data_ptr());
    c.v_scale = static_cast<float*>(vs.data_ptr());
    c.pages = k.size(0);
    c.heads = (int)k.size(1);
    c.page = (int)k.size(2);
    c.head_dim = (int)k.size(3);
    return c;
}
struct Table {
    const int32_t* p;
    int64_t ld, width;
    int batch;
    explicit Table(PyObject* o) {
        const at::Tensor& t = on_device(rowmajor(o), "the page table");
        if (t.scalar_type() != at::kInt || t.size(0) > 0x7fffffff) {
            PyErr_SetString(PyExc_ValueError, "the page table has to be int32");
            throw Refused();
        }
        p = static_cast<int32_t*>(t.data_ptr());
        width = t.size(1);
        ld = t.size(0) > 1 ? t.stride(0) : width;
        batch = (int)t.size(0);
    }
};

// kv8_append(k, v, cache k, v, k_scale, v_scale, table, kv_len, offsets, max_new) -> None
PyObject* kv8_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 10);
        const fq_kv8_cache cache = cache_of(a + 2);
        const int64_t width = (int64_t)cache.heads * cache.head_dim;
        const at::Tensor &k = rows_of(a[0], width, "k"), &v = rows_of(a[1], width, "v");
        if (v.size(0) != k.size(0) || v.scalar_type() != k.scalar_type()) {
            PyErr_SetString(PyExc_ValueError, "k and v have to have the same rows and dtype");
            throw Refused();
        }
        const fq_dtype xt = dtype_of(k.scalar_type());
        const Table t(a[6]);
        const int32_t* kv_len = static_cast<int32_t*>(vector_of(a[7], at::kInt, t.batch, "kv_len").data_ptr());
        const int32_t* offsets = data_or_null<int32_t>(a[8], at::kInt, (int64_t)t.batch + 1, "offsets");
        const int64_t max_new = integer(a[9]);
        fq_status s;
        {
            const Unlocked nogil;
            s = fq_kv8_append(k.data_ptr(), v.data_ptr(), xt, k.size(0), pitch(k), pitch(v), &cache, t.p, t.ld, t.width, t.batch, kv_len, offsets, max_new, stream());
        }
        if (s != FQ_OK) return status(s);
        Py_RETURN_NONE;
    });
}

// attention_kv8(q, q_heads, cache k, v, k_scale, v_scale, table, kv_len, offsets, max_q, max_kv, causal, scale, y, workspace)
PyObject* attention_kv8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 15);
        const int64_t q_heads = integer(a[1]);
        const fq_kv8_cache cache = cache_of(a + 2);
        if (q_heads < 1 || q_heads > 65535) return status(q_heads < 1 ? FQ_ERR_INVALID_ARG : FQ_ERR_UNSUPPORTED);
        const int64_t width = q_heads * cache.head_dim;
        const at::Tensor& q = rows_of(a[0], width, "q");
        const fq_dtype dt = dtype_of(q.scalar_type());
        const Table t(a[6]);
        const int32_t* kv_len = static_cast<int32_t*>(vector_of(a[7], at::kInt, t.batch, "kv_len").data_ptr());
        const int32_t* offsets = data_or_null<int32_t>(a[8], at::kInt, (int64_t)t.batch + 1, "offsets");
        const int64_t max_q = integer(a[9]), max_kv = integer(a[10]);
        const int causal = integer(a[11]) != 0;
        const float scale = real(a[12]);
        RowsOut y(a[13], q.size(0), width, q.scalar_type(), "y");
        if (!none(a[14])) on_device(tensor(a[14]), "the workspace");
        Workspace ws(a[14]);
        fq_status s;
        {
            const Unlocked nogil;
            y.make(q.size(0), width, q.scalar_type(), q);
            ws.make([&] { return fq_attention_kv8_workspace_bytes(dt, q.size(0), (int)q_heads, &cache, t.width, t.batch, offsets != nullptr, max_q, max_kv); }, q);
            s = fq_attention_kv8(q.data_ptr(), dt, q.size(0), pitch(q), (int)q_heads, &cache, t.p, t.ld, t.width, t.batch, kv_len, offsets, max_q, max_kv,
                                 causal, scale, y.t.data_ptr(), pitch(y.t), ws.p, ws.bytes, stream());
        }
        return s == FQ_OK ? THPVariable_Wrap(std::move(y.t)) : status(s);
    });
}

// cross_attention(q, k, v, q_heads, kv_heads, batch, q_offsets, kv_offsets, kv_len, key_mask, max_q, max_kv, scale, y, workspace)
PyObject* cross_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 15);
        const int64_t q_heads = integer(a[3]), kv_heads = integer(a[4]), batch = integer(a[5]);
        if (q_heads < 1 || kv_heads < 1 || batch < 0) return status(FQ_ERR_INVALID_ARG);
        if (q_heads > 65535 || kv_heads > 65535 || batch > 65535) return status(FQ_ERR_UNSUPPORTED);
        const at::Tensor& q = on_device(rowmajor(a[0]), "q");
        const int64_t width = q.size(1), D = width / q_heads;
        if (D * q_heads != width) return status(FQ_ERR_INVALID_ARG);
        const at::Tensor &k = rows_of(a[1], kv_heads * D, "k"), &v = rows_of(a[2], kv_heads * D, "v");
        if (v.size(0) != k.size(0) || k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type()) {
            PyErr_SetString(PyExc_ValueError, "k and v have to have the same rows, and the dtype of q");
            throw Refused();
        }
        const fq_dtype dt = dtype_of(q.scalar_type());
        const int32_t* q_offsets = data_or_null<int32_t>(a[6], at::kInt, batch + 1, "q_offsets");
        const int32_t* kv_offsets = data_or_null<int32_t>(a[7], at::kInt, batch + 1, "kv_offsets");
        const int32_t* kv_len = data_or_null<int32_t>(a[8], at::kInt, batch, "kv_len");
        const uint8_t* mask = nullptr;
        if (!none(a[9])) {
            const at::Tensor& m = on_device(tensor(a[9]), "key_mask");
            if ((m.scalar_type() != at::kBool && m.scalar_type() != at::kByte) || !m.is_contiguous() || m.numel() != k.size(0)) {
                PyErr_SetString(PyExc_ValueError, "key_mask has to be a contiguous bool or uint8 tensor with an element for each row of k");
                throw Refused();
            }
            mask = static_cast<const uint8_t*>(m.data_ptr());
        }
        const int64_t max_q = integer(a[10]), max_kv = integer(a[11]);
        const float scale = real(a[12]);
        RowsOut y(a[13], q.size(0), width, q.scalar_type(), "y");
        if (!none(a[14])) on_device(tensor(a[14]), "the workspace");
        Workspace ws(a[14]);
        fq_status s;
        {
            const Unlocked nogil;
            y.make(q.size(0), width, q.scalar_type(), q);
            ws.make([&] { return fq_cross_attention_workspace_bytes(dt, q.size(0), (int)q_heads, k.size(0), (int)kv_heads, (int)D, (int)batch, q_offsets != nullptr, kv_offsets != nullptr, max_q, max_kv); }, q);
            s = fq_cross_attention(q.data_ptr(), dt, q.size(0), pitch(q), (int)q_heads, k.data_ptr(), v.data_ptr(), k.size(0), pitch(k), pitch(v), (int)kv_heads,
                                   (int)D, (int)batch, q_offsets, kv_offsets, kv_len, mask, max_q, max_kv, scale, y.t.data_ptr(), pitch(y.t), ws.p, ws.bytes, stream());
        }
        return s == FQ_OK ? THPVariable_Wrap(std::move(y.t)) : status(s);
    });
}

// ---- projections in microscaled 4-bit floating point, norms that end in codes ----
// A contiguous tensor of `bytes` bytes or float elements: the caller's, or a new one of `size`.
struct FlatOut {
    at::Tensor t;
    FlatOut(PyObject* given, at::ScalarType type, int64_t count, const char* what) {
        if (none(given)) return;
        t = on_device(tensor(given), what);
        if (t.scalar_type() != type || !t.is_contiguous() || t.numel() != count) {
            PyErr_Format(PyExc_ValueError, "%s has to be a contiguous %s tensor of %lld elements", what, at::toString(type), (long long)count);
            throw Refused();
        }
    }
    template <typename T = void>
    T* data() { return static_cast<T*>(t.data_ptr()); }
};
// Outputs of one call that nobody brought, in one allocation, each from a multiple of 256 bytes on: codes, scales and steps go from call to
// call together, and three allocations cost as much host time as a launch (50 x 1024 into NVFP4: 5.4 us a call, so 4.5).
struct Together {
    int64_t bytes = 0;
    struct Part {
        FlatOut* out;
        at::DimVector size;
        at::ScalarType type;
        int64_t at;
    };
    c10::SmallVector<Part, 4> parts;
    void add(FlatOut& out, at::IntArrayRef size, at::ScalarType type) {
        if (out.t.defined()) return;
        int64_t n = static_cast<int64_t>(c10::elementSize(type));
        for (int64_t d : size) n *= d;
        parts.push_back({&out, at::DimVector(size.begin(), size.end()), type, bytes});
        bytes += (n + 255) / 256 * 256;
    }
    void make(const at::Tensor& like) {
        if (parts.empty()) return;
        const at::Tensor all = fresh({bytes}, at::kByte, like);
        for (const Part& p : parts) {
            at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(p.type));
            t.unsafeGetTensorImpl()->set_storage_offset(p.at / static_cast<int64_t>(c10::elementSize(p.type)));
            t.unsafeGetTensorImpl()->set_sizes_contiguous(p.size);
            p.out->t = std::move(t);
        }
    }
};
PyObject* tuple_of(std::initializer_list<at::Tensor> list) {
    PyObject* r = PyTuple_New((Py_ssize_t)list.size());
    if (!r) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : list) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));
    return r;
}
// A site's multiplier: None (the constant block^-1/2), a float tensor of K elements, or the address of a handle's own.
const float* multiplier_of(PyObject* o, int64_t K) {
    if (none(o)) return nullptr;
    if (PyLong_Check(o)) return static_cast<const float*>(address(o));
    return static_cast<const float*>(vector_of(o, at::kFloat, K, "mult_g").data_ptr());
}
fq_fp4_format format_of(long long f) { return f == FQ_MXFP4 || f == FQ_NVFP4 ? static_cast<fq_fp4_format>(f) : static_cast<fq_fp4_format>(7); }
bool known(fq_fp4_format f) { return f == FQ_MXFP4 || f == FQ_NVFP4; }

// quantize_act_fp4(x, multiplier, block, format, codes, scales, delta) -> (codes, scales, delta)
PyObject* quantize_act_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 7);
        const at::Tensor& x = on_device(rowmajor(a[0]), "x");
        const int64_t M = x.size(0), K = x.size(1);
        const float* g = multiplier_of(a[1], K);
        const long long block = integer(a[2]);
        const fq_fp4_format f = format_of(integer(a[3]));
        const fq_dtype xt = dtype_of(x.scalar_type());
        if (!known(f)) return status(FQ_ERR_INVALID_ARG);
        const int64_t sb = (int64_t)fq_fp4_scale_bytes(M, K, f);
        FlatOut codes(a[4], at::kByte, M * (K / 2), "codes"), scales(a[5], at::kByte, sb, "scales"), delta(a[6], at::kFloat, M, "delta");
        fq_status s;
        {
            const Unlocked nogil;
            Together outs;
            outs.add(codes, {M, K / 2}, at::kByte);
            outs.add(scales, {sb}, at::kByte);
            outs.add(delta, {M}, at::kFloat);
            outs.make(x);
            s = fq_quantize_act_fp4(x.data_ptr(), xt, M, K, pitch(x), g, block == (int)block ? (int)block : 0, f, codes.data(), scales.data(),
                                    delta.data<float>(), stream());
        }
        return s == FQ_OK ? tuple_of({codes.t, scales.t, delta.t}) : status(s);
    });
}

// gemm_fp4(codes, scales, delta, handle, K, N, format, out_dtype, y)
PyObject* gemm_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 9);
        const fq_fp4_weights* W = static_cast<const fq_fp4_weights*>(address(a[3]));
        const int64_t K = integer(a[4]), N = integer(a[5]);
        const fq_fp4_format f = format_of(integer(a[6]));
        const at::Tensor& codes = rows_of(a[0], K / 2, "codes");
        const int64_t M = codes.size(0);
        if (codes.scalar_type() != at::kByte || !codes.is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "codes have to be contiguous uint8");
            throw Refused();
        }
        const at::Tensor& scales = vector_of(a[1], at::kByte, (int64_t)fq_fp4_scale_bytes(M, K, f), "scales");
        const at::Tensor& delta = vector_of(a[2], at::kFloat, M, "delta");
        Output type(a[8], a[7]);
        RowsOut y(a[8], M, N, type.type, "y");
        fq_status s;
        {
            const Unlocked nogil;
            y.make(M, N, type.type, codes);
            s = fq_gemm_fp4(codes.data_ptr(), scales.data_ptr(), static_cast<const float*>(delta.data_ptr()), M, W, y.t.data_ptr(), type.dt, pitch(y.t),
                            stream());
        }
        return s == FQ_OK ? THPVariable_Wrap(std::move(y.t)) : status(s);
    });
}

// linear_fp4(x, handle, K, N, format, out_dtype, y, workspace)
PyObject* linear_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 8);
        const fq_fp4_weights* W = static_cast<const fq_fp4_weights*>(address(a[1]));
        const int64_t K = integer(a[2]), N = integer(a[3]);
        const fq_fp4_format f = format_of(integer(a[4]));
        const at::Tensor& x = rows_of(a[0], K, "x");
        const int64_t M = x.size(0);
        const fq_dtype xt = dtype_of(x.scalar_type());
        Output type(a[6], a[5]);
        RowsOut y(a[6], M, N, type.type, "y");
        void* wp = nullptr;
        size_t wbytes = 0;
        if (!none(a[7])) {
            const at::Tensor& t = on_device(tensor(a[7]), "workspace");
            if (t.scalar_type() != at::kByte || !t.is_contiguous()) {
                PyErr_SetString(PyExc_ValueError, "workspace has to be contiguous uint8");
                throw Refused();
            }
            wp = t.data_ptr();
            wbytes = static_cast<size_t>(t.numel());
        }
        const bool given = !none(a[7]);
        fq_status s;
        {
            const Unlocked nogil;
            y.make(M, N, type.type, x);
            c10::DataPtr own;                // (for the length of the call, as Workspace, without a tensor around it)
            if (!given) {
                wbytes = fq_linear_fp4_workspace_bytes(M, K, f);
                own = c10::cuda::CUDACachingAllocator::get()->allocate(wbytes);
                wp = own.get();
            }
            s = fq_linear_fp4(x.data_ptr(), xt, M, pitch(x), W, y.t.data_ptr(), type.dt, pitch(y.t), wp, wbytes, stream());
        }
        return s == FQ_OK ? THPVariable_Wrap(std::move(y.t)) : status(s);
    });
}

// What the two norms share: x, residual and the stream that they add up to.
struct NormRows {
    const at::Tensor& x;
    const at::Tensor* residual;
    int64_t M, K;
    fq_dtype xt;
    RowsOut h;
    NormRows(PyObject* xo, PyObject* ro, PyObject* ho)
        : x(on_device(rowmajor(xo), "x")), residual(none(ro) ? nullptr : &rows_of(ro, x.size(1), "residual")), M(x.size(0)), K(x.size(1)),
          xt(dtype_of(x.scalar_type())), h(ho, x.size(0), x.size(1), x.scalar_type(), "h") {
        if (residual && (residual->size(0) != M || residual->scalar_type() != x.scalar_type())) {
            PyErr_SetString(PyExc_ValueError, "x and residual have to have the same rows and dtype");
            throw Refused();
        }
        if (!residual && h.t.defined()) {
            PyErr_SetString(PyExc_ValueError, "h is written where there is a residual");
            throw Refused();
        }
    }
    void make() { if (residual) h.make(M, K, x.scalar_type(), x); }
    const void* rp() const { return residual ? residual->data_ptr() : nullptr; }
    int64_t ldr() const { return residual ? pitch(*residual) : 0; }
    void* hp() { return residual ? h.t.data_ptr() : nullptr; }
    int64_t ldh() { return residual ? pitch(h.t) : 0; }
    const at::Tensor& stream_rows() { return residual ? h.t : x; }
};

// rmsnorm_quantize_act(x, residual, multiplier, block, bits, eps, clip_ratio, h, codes, delta) -> (h, codes, delta)
PyObject* rmsnorm_quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 10);
        NormRows r(a[0], a[1], a[7]);
        const float* g = multiplier_of(a[2], r.K);
        const long long block = integer(a[3]), bits = integer(a[4]);
        const float eps = real(a[5]), clip = real(a[6]);
        if (bits != 4 && bits != 8) return status(FQ_ERR_INVALID_ARG);
        FlatOut codes(a[8], at::kByte, r.M * (r.K * bits / 8), "codes"), delta(a[9], at::kFloat, r.M, "delta");
        fq_status s;
        {
            const Unlocked nogil;
            r.make();
            Together outs;
            outs.add(codes, {r.M, r.K * bits / 8}, at::kByte);
            outs.add(delta, {r.M}, at::kFloat);
            outs.make(r.x);
            s = fq_rmsnorm_quantize_act(r.x.data_ptr(), r.rp(), r.xt, r.M, r.K, pitch(r.x), r.ldr(), eps, r.hp(), r.ldh(), g,
                                        block == (int)block ? (int)block : 0, (int)bits, clip, codes.data(), delta.data<float>(), stream());
        }
        return s == FQ_OK ? tuple_of({r.stream_rows(), codes.t, delta.t}) : status(s);
    });
}

// rmsnorm_quantize_act_fp4(x, residual, multiplier, block, format, eps, h, codes, scales, delta) -> (h, codes, scales, delta)
PyObject* rmsnorm_quantize_act_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 10);
        NormRows r(a[0], a[1], a[6]);
        const float* g = multiplier_of(a[2], r.K);
        const long long block = integer(a[3]);
        const fq_fp4_format f = format_of(integer(a[4]));
        const float eps = real(a[5]);
        if (!known(f)) return status(FQ_ERR_INVALID_ARG);
        const int64_t sb = (int64_t)fq_fp4_scale_bytes(r.M, r.K, f);
        FlatOut codes(a[7], at::kByte, r.M * (r.K / 2), "codes"), scales(a[8], at::kByte, sb, "scales"), delta(a[9], at::kFloat, r.M, "delta");
        fq_status s;
        {
            const Unlocked nogil;
            r.make();
            Together outs;
            outs.add(codes, {r.M, r.K / 2}, at::kByte);
            outs.add(scales, {sb}, at::kByte);
            outs.add(delta, {r.M}, at::kFloat);
            outs.make(r.x);
            s = fq_rmsnorm_quantize_act_fp4(r.x.data_ptr(), r.rp(), r.xt, r.M, r.K, pitch(r.x), r.ldr(), eps, r.hp(), r.ldh(), g,
                                            block == (int)block ? (int)block : 0, f, codes.data(), scales.data(), delta.data<float>(), stream());
        }
        return s == FQ_OK ? tuple_of({r.stream_rows(), codes.t, scales.t, delta.t}) : status(s);
    });
}

#define FQ_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FQ_METHOD(linear), FQ_METHOD(linear_gated), FQ_METHOD(gemm), FQ_METHOD(quantize_act), FQ_METHOD(quantize_act_composite),
                         FQ_METHOD(linear_w4a16), FQ_METHOD(qk_norm_rope), FQ_METHOD(kv8_append),
                         FQ_METHOD(attention_kv8), FQ_METHOD(cross_attention), FQ_METHOD(quantize_act_fp4), FQ_METHOD(gemm_fp4),
                         FQ_METHOD(linear_fp4), FQ_METHOD(rmsnorm_quantize_act), FQ_METHOD(rmsnorm_quantize_act_fp4), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fq_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fq_torch(void) { return PyModule_Create(&module); }
