// The hot calls of the Python binding in native code: argument checks, marshalling and the call into
// librtn for one entry point each.  A pass over a network's layers at batch 1 is bound by the host, and
// the same work through ctypes took 6 to 10 us per call (it takes about 1 us here); the GPU needs 4 to
// 8 us for such a layer.  binding.py keeps the public signatures, allocates default outputs and
// raises on a status; the checks below raise what it raised: AssertionError for a tensor of the
// wrong device, type or layout, ValueError for a code tensor that does not hold the stated codes.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/rtn.h"

namespace {

// Thrown after a Python error has been set.
struct PyError {};

[[noreturn]] void fail(PyObject* type, const char* fmt, const char* what)
{
    PyErr_Format(type, fmt, what);
    throw PyError();
}

int64_t integer(PyObject* o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PyError();
    return v;
}
int truth(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PyError();
    return v;
}

const at::Tensor& tensor(PyObject* o, const char* what)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s: a torch tensor is required", what);
    return THPVariable_Unpack(o);
}

// Data pointer of a contiguous device tensor of the given type; None -> NULL.
void* dev(PyObject* o, c10::ScalarType type, const char* what, bool nullable = true)
{
    if (nullable && o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, what);
    if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous())
        fail(PyExc_AssertionError, "%s: a contiguous device tensor of the documented type is required", what);
    return t.data_ptr();
}
// Any tensor's storage, unchecked (workspaces, prepared weights).
void* raw(PyObject* o, const char* what) { return o == Py_None ? nullptr : tensor(o, what).data_ptr(); }
size_t raw_bytes(PyObject* o, const char* what) { return o == Py_None ? 0 : tensor(o, what).nbytes(); }

// The library takes raw pointers: make sure the tensor really holds `rows` rows of K codes in format
// fmt, so that a tensor packed in another format cannot be read out of bounds.
void* codes(PyObject* o, int64_t rows, int64_t K, rtn_code_format fmt, const char* what)
{
    const at::Tensor& t = tensor(o, what);
    const size_t need = rtn_codes_bytes(fmt, rows, K), have = t.nbytes();
    if (!(t.is_cuda() && t.is_contiguous() && have >= need)) {
        PyErr_Format(PyExc_ValueError, "%s: %zu bytes, but %lld rows of %lld codes in format %d need %zu", what, have,
                     (long long)rows, (long long)K, (int)fmt, need);
        throw PyError();
    }
    const c10::ScalarType type = t.scalar_type();
    if ((fmt == RTN_CODE_FP4 && type != c10::kByte) || (fmt == RTN_CODE_I8 && type != c10::kChar) ||
        (fmt == RTN_CODE_BITPLANE && type != c10::kLong && type != c10::kUInt64))
        fail(PyExc_ValueError, "%s: dtype does not match the code format", what);
    return t.data_ptr();
}

// A python number (host scalar) or a device float32 vector.
struct Gran {
    float s = 0.0f;
    const float* ptr = nullptr;
    rtn_gran gran = RTN_SCALAR;
    Gran(PyObject* o, const char* what)
    {
        if (o == Py_None) return;
        if (THPVariable_Check(o)) {
            ptr = (const float*)dev(o, c10::kFloat, what, false);
            gran = RTN_VECTOR;
        } else {
            const double v = PyFloat_AsDouble(o);
            if (v == -1.0 && PyErr_Occurred()) throw PyError();
            s = (float)v;
            ptr = &s;
        }
    }
    Gran(const Gran&) = delete;
};

const rtn_epilogue* epilogue(PyObject* o)  // address of an Epilogue's struct, or None
{
    if (o == Py_None) return nullptr;
    const void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw PyError();
    return (const rtn_epilogue*)p;
}

// torch's current stream.  On a host without a GPU the library's own checks must be what raises.
void* stream()
{
    try {
        return (void*)c10::hip::getCurrentHIPStream().stream();
    } catch (const c10::Error&) {
        if (c10::hip::device_count() > 0) throw;
        return nullptr;
    }
}

// The interpreter's lock is given up around a call into the library, as ctypes gives it up: a launch that
// loads its code object or waits for room in the queue must not stop every other Python thread.  The
// arguments are converted before (the caller's frame keeps them alive meanwhile).
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// Runs `f` on the arguments; a C++ exception or a wrong argument count becomes a Python error, and torch's of a full
// device torch.OutOfMemoryError.
template <class F>
PyObject* call(Py_ssize_t want, Py_ssize_t n, F f)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
        return nullptr;
    }
    try {
        return PyLong_FromLong(f());
    } catch (const PyError&) {
        return nullptr;
    } catch (const c10::OutOfMemoryError&) {
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
typedef PyObject* const* Args;

// x, layout, d0, d1, d2, d3, lo, hi, fmt, codes, sum_t
PyObject* pack(PyObject*, Args a, Py_ssize_t n)
{
    return call(11, n, [&] {
        const Gran lo(a[6], "lo"), hi(a[7], "hi");
        if (lo.gran != hi.gran) fail(PyExc_AssertionError, "%s: lo and hi must both be scalars or both vectors", "ternarize_pack");
        const float* x = (const float*)dev(a[0], c10::kFloat, "x");
        const rtn_layout layout = (rtn_layout)integer(a[1]);
        const int64_t d0 = integer(a[2]), d1 = integer(a[3]), d2 = integer(a[4]), d3 = integer(a[5]);
        const rtn_code_format fmt = (rtn_code_format)integer(a[8]);
        void* out = raw(a[9], "codes");
        int32_t* sum = (int32_t*)dev(a[10], c10::kInt, "sum_t");
        void* st = stream();
        const Unlocked u;
        return rtn_ternarize_pack(x, layout, d0, d1, d2, d3, lo.ptr, hi.ptr, lo.gran, fmt, out, sum, st);
    });
}

// fmt, path, a_codes, w_codes, M, N, K, acc_out, ep, y_out
PyObject* gemm(PyObject*, Args a, Py_ssize_t n)
{
    return call(10, n, [&] {
        const rtn_code_format fmt = (rtn_code_format)integer(a[0]);
        const rtn_path path = (rtn_path)integer(a[1]);
        const int64_t M = integer(a[4]), N = integer(a[5]), K = integer(a[6]);
        const void *ac = codes(a[2], M, K, fmt, "a_codes"), *wc = codes(a[3], N, K, fmt, "w_codes");
        int32_t* acc = (int32_t*)dev(a[7], c10::kInt, "acc_out");
        const rtn_epilogue* ep = epilogue(a[8]);
        float* y = (float*)dev(a[9], c10::kFloat, "y_out");
        void* st = stream();
        const Unlocked u;
        return rtn_ternary_gemm(fmt, path, ac, wc, M, N, K, acc, ep, y, nullptr, 0, st);
    });
}

// fmt, path, a_codes, w_codes, Nb, C, H, W, O, KH, KW, stride, pad, pad_mode, acc_out, ep, y_out, workspace
PyObject* conv2d(PyObject*, Args a, Py_ssize_t n)
{
    return call(18, n, [&] {
        const rtn_code_format fmt = (rtn_code_format)integer(a[0]);
        const rtn_path path = (rtn_path)integer(a[1]);
        const int64_t Nb = integer(a[4]), C = integer(a[5]), H = integer(a[6]), W = integer(a[7]), O = integer(a[8]);
        const int KH = (int)integer(a[9]), KW = (int)integer(a[10]), stride = (int)integer(a[11]), pad = (int)integer(a[12]);
        const rtn_pad_mode mode = (rtn_pad_mode)integer(a[13]);
        const void* ac = codes(a[2], Nb * H * W, C, fmt, "a_codes");
        const void* wc = codes(a[3], O * KH * KW, C, fmt, "w_codes");
        int32_t* acc = (int32_t*)dev(a[14], c10::kInt, "acc_out");
        const rtn_epilogue* ep = epilogue(a[15]);
        float* y = (float*)dev(a[16], c10::kFloat, "y_out");
        void* ws = raw(a[17], "workspace");
        const size_t wsb = raw_bytes(a[17], "workspace");
        void* st = stream();
        const Unlocked u;
        return rtn_ternary_conv2d_implicit_gemm(fmt, path, ac, wc, Nb, C, H, W, O, KH, KW, stride, pad, mode, acc, ep, y, ws, wsb, st);
    });
}

// fmt, path, a_codes, w_codes, Nb, C, H, W, O, KH, KW, stride, pad, pad_mode, ep, residual, relu_out, lo, hi, y_out, codes_out,
// workspace
PyObject* conv2d_ternarize(PyObject*, Args a, Py_ssize_t n)
{
    return call(22, n, [&] {
        const rtn_code_format fmt = (rtn_code_format)integer(a[0]);
        const rtn_path path = (rtn_path)integer(a[1]);
        const int64_t Nb = integer(a[4]), C = integer(a[5]), H = integer(a[6]), W = integer(a[7]), O = integer(a[8]);
        const int KH = (int)integer(a[9]), KW = (int)integer(a[10]), stride = (int)integer(a[11]), pad = (int)integer(a[12]);
        const rtn_pad_mode mode = (rtn_pad_mode)integer(a[13]);
        const void* ac = codes(a[2], Nb * H * W, C, fmt, "a_codes");
        const void* wc = codes(a[3], O * KH * KW, C, fmt, "w_codes");
        const int64_t OH = stride > 0 ? (H + 2 * pad - KH) / stride + 1 : 0, OW = stride > 0 ? (W + 2 * pad - KW) / stride + 1 : 0;
        void* co = codes(a[20], Nb * OH * OW, O, fmt, "codes_out");
        const Gran lo(a[17], "lo"), hi(a[18], "hi");
        if (lo.gran != hi.gran) fail(PyExc_AssertionError, "%s: lo and hi must both be scalars or both vectors", "ternary_conv2d_ternarize");
        const rtn_epilogue* ep = epilogue(a[14]);
        const float* res = (const float*)dev(a[15], c10::kFloat, "residual");
        const int relu_out = truth(a[16]);
        float* y = (float*)dev(a[19], c10::kFloat, "y_out");
        void* ws = raw(a[21], "workspace");
        const size_t wsb = raw_bytes(a[21], "workspace");
        void* st = stream();
        const Unlocked u;
        return rtn_ternary_conv2d_ternarize(fmt, path, ac, wc, Nb, C, H, W, O, KH, KW, stride, pad, mode, ep, res, relu_out, lo.ptr, hi.ptr,
                                            lo.gran, y, co, ws, wsb, st);
    });
}

// a_codes, w_codes, Nb, C, H, W, KH, KW, stride, pad, pad_mode, acc_out, ep, y_out
PyObject* depthwise(PyObject*, Args a, Py_ssize_t n)
{
    return call(14, n, [&] {
        const int64_t Nb = integer(a[2]), C = integer(a[3]), H = integer(a[4]), W = integer(a[5]);
        const int KH = (int)integer(a[6]), KW = (int)integer(a[7]), stride = (int)integer(a[8]), pad = (int)integer(a[9]);
        const rtn_pad_mode mode = (rtn_pad_mode)integer(a[10]);
        const void* ac = codes(a[0], Nb * H * W, C, RTN_CODE_I8, "a_codes");
        const void* wc = codes(a[1], C, KH * KW, RTN_CODE_I8, "w_codes");
        int32_t* acc = (int32_t*)dev(a[11], c10::kInt, "acc_out");
        const rtn_epilogue* ep = epilogue(a[12]);
        float* y = (float*)dev(a[13], c10::kFloat, "y_out");
        void* st = stream();
        const Unlocked u;
        return rtn_ternary_depthwise_conv2d(ac, wc, Nb, C, H, W, KH, KW, stride, pad, mode, acc, ep, y, st);
    });
}

// x, w_codes or prepared, is_prepared, M, N, K, alpha_w, relu, bn_scale, bn_shift, y_out, workspace
PyObject* weight_gemm(PyObject*, Args a, Py_ssize_t n)
{
    return call(12, n, [&] {
        const Gran al(a[6], "alpha_w");
        auto fn = truth(a[2]) ? rtn_ternary_weight_gemm_prepared : rtn_ternary_weight_gemm;
        const float* x = (const float*)dev(a[0], c10::kFloat, "x");
        const void* w = raw(a[1], "w_codes");
        const int64_t M = integer(a[3]), N = integer(a[4]), K = integer(a[5]);
        const int relu = truth(a[7]);
        const float *bs = (const float*)dev(a[8], c10::kFloat, "bn_scale"), *bh = (const float*)dev(a[9], c10::kFloat, "bn_shift");
        float* y = (float*)dev(a[10], c10::kFloat, "y_out");
        void* ws = raw(a[11], "workspace");
        const size_t wsb = raw_bytes(a[11], "workspace");
        void* st = stream();
        const Unlocked u;
        return fn(x, w, M, N, K, al.ptr, al.gran, relu, bs, bh, y, ws, wsb, st);
    });
}

// x, prepared, Nb, C, H, W, O, KH, KW, stride, pad, relu, y_out, workspace
PyObject* weight_conv2d_prepared(PyObject*, Args a, Py_ssize_t n)
{
    return call(14, n, [&] {
        const float* x = (const float*)dev(a[0], c10::kFloat, "x");
        const void* w = raw(a[1], "prepared");
        const int64_t Nb = integer(a[2]), C = integer(a[3]), H = integer(a[4]), W = integer(a[5]), O = integer(a[6]);
        const int KH = (int)integer(a[7]), KW = (int)integer(a[8]), stride = (int)integer(a[9]), pad = (int)integer(a[10]);
        const int relu = truth(a[11]);
        float* y = (float*)dev(a[12], c10::kFloat, "y_out");
        void* ws = raw(a[13], "workspace");
        const size_t wsb = raw_bytes(a[13], "workspace");
        void* st = stream();
        const Unlocked u;
        return rtn_ternary_weight_conv2d_prepared(x, w, Nb, C, H, W, O, KH, KW, stride, pad, relu, y, ws, wsb, st);
    });
}

// a, grad_out, n, lo, hi, gamma, grad_in, sums, workspace
PyObject* activation_backward(PyObject*, Args a, Py_ssize_t n)
{
    return call(9, n, [&] {
        const Gran lo(a[3], "lo"), hi(a[4], "hi"), ga(a[5], "gamma");
        const float *x = (const float*)dev(a[0], c10::kFloat, "a"), *g = (const float*)dev(a[1], c10::kFloat, "grad_out");
        const int64_t count = integer(a[2]);
        float* gi = (float*)dev(a[6], c10::kFloat, "grad_in");
        double* sums = (double*)dev(a[7], c10::kDouble, "sums");
        void* ws = raw(a[8], "workspace");
        const size_t wsb = raw_bytes(a[8], "workspace");
        void* st = stream();
        const Unlocked u;
        return rtn_activation_backward(x, g, count, lo.ptr, hi.ptr, ga.ptr, gi, sums, ws, wsb, st);
    });
}

// w, grad_out, O, K, lo, hi, k_w, b_w, alpha, grad_w, sums
PyObject* weight_backward(PyObject*, Args a, Py_ssize_t n)
{
    return call(11, n, [&] {
        const Gran lo(a[4], "lo"), hi(a[5], "hi");
        const float *w = (const float*)dev(a[0], c10::kFloat, "w"), *g = (const float*)dev(a[1], c10::kFloat, "grad_out");
        const int64_t O = integer(a[2]), K = integer(a[3]);
        const float *kw = (const float*)dev(a[6], c10::kFloat, "k_w"), *bw = (const float*)dev(a[7], c10::kFloat, "b_w"),
                    *al = (const float*)dev(a[8], c10::kFloat, "alpha");
        float* gw = (float*)dev(a[9], c10::kFloat, "grad_w");
        double* sums = (double*)dev(a[10], c10::kDouble, "sums");
        void* st = stream();
        const Unlocked u;
        return rtn_weight_backward(w, g, O, K, lo.ptr, hi.ptr, kw, bw, al, gw, sums, st);
    });
}

// Bytes or a matrix on the device of `like`.
at::Tensor make_bytes(size_t n, const at::Tensor& like) { return at::empty({(int64_t)n}, like.options().dtype(c10::kByte)); }
at::Tensor make_rows(int64_t rows, int64_t cols, c10::ScalarType type, const at::Tensor& like)
{
    return at::empty({rows, cols}, like.options().dtype(type));
}
// `given`, or what `make` allocates where it is None
template <class F>
at::Tensor given_or(PyObject* given, const char* what, F make)
{
    return given == Py_None ? make() : tensor(given, what);
}
void* rows2d(const at::Tensor& t, c10::ScalarType type, int64_t rows, int64_t len, const char* what, int64_t& ld)
{
    if (!t.is_cuda() || t.scalar_type() != type || t.dim() != 2 || t.size(0) != rows || t.size(1) != len ||
        (len > 1 && t.stride(1) != 1))
        fail(PyExc_AssertionError, "%s: a device tensor of the documented type and shape, its rows dense, is required", what);
    ld = rows > 1 ? t.stride(0) : len;
    return t.data_ptr();
}
void* bytes_of(const at::Tensor& t, size_t need, const char* what)
{
    if (!(t.is_cuda() && t.is_contiguous() && t.nbytes() >= need)) {
        PyErr_Format(PyExc_ValueError, "%s: a device buffer of %zu bytes is required", what, need);
        throw PyError();
    }
    return t.data_ptr();
}
// A workspace: the kernels write all over it (its size is the library's to check).
void* scratch(const at::Tensor& t)
{
    if (!t.is_cuda() || !t.is_contiguous()) fail(PyExc_ValueError, "%s: a contiguous device buffer is required", "workspace");
    return t.data_ptr();
}
void* rows2d(PyObject* o, c10::ScalarType type, int64_t rows, int64_t len, const char* what, int64_t& ld)
{
    ld = len;
    return o == Py_None ? nullptr : rows2d(tensor(o, what), type, rows, len, what, ld);
}
void* bytes_of(PyObject* o, size_t need, const char* what) { return o == Py_None ? nullptr : bytes_of(tensor(o, what), need, what); }
void* vector_of(PyObject* o, c10::ScalarType type, int64_t n, const char* what)
{
    void* p = dev(o, type, what);
    if (p && tensor(o, what).numel() != n) fail(PyExc_AssertionError, "%s: one entry per output is required", what);
    return p;
}
rtn_dtype dtype(c10::ScalarType t, const char* what, bool f32 = false)
{
    if (t == c10::kBFloat16) return RTN_BF16;
    if (t == c10::kHalf) return RTN_F16;
    if (!f32 || t != c10::kFloat) fail(PyExc_AssertionError, "%s: bfloat16 or float16 is required", what);
    return RTN_F32;
}
const at::Tensor& matrix(PyObject* o, const char* what)
{
    const at::Tensor& t = tensor(o, what);
    if (!t.is_cuda() || t.dim() != 2) fail(PyExc_AssertionError, "%s: a matrix on the device is required", what);
    return t;
}
struct AlphaN : Gran {
    AlphaN(PyObject* o, int64_t n) : Gran(o, "alpha_w")
    {
        if (gran == RTN_VECTOR && tensor(o, "alpha_w").numel() != n) fail(PyExc_AssertionError, "%s: one entry per output is required", "alpha_w");
    }
};

// Runs `f`, which returns a status and leaves its outputs; on RTN_OK the outputs are the result (one, or a tuple with None for
// what is undefined), else the status.
template <int N, class F>
PyObject* call_for(Py_ssize_t want, Py_ssize_t n, F f)
{
    at::Tensor out[N];
    PyObject* status = call(want, n, [&] { return f(out); });
    if (!status || PyLong_AsLong(status) != RTN_OK) return status;
    Py_DECREF(status);
    auto wrap = [](at::Tensor& t) -> PyObject* { return t.defined() ? THPVariable_Wrap(std::move(t)) : Py_NewRef(Py_None); };
    if (N == 1) return wrap(out[0]);
    PyObject* tuple = PyTuple_New(N);
    for (int i = 0; tuple && i < N; ++i) PyTuple_SET_ITEM(tuple, i, wrap(out[i]));
    return tuple;
}

// w_codes, N, K, fmt, backward
PyObject* linear_prepare(PyObject*, Args a, Py_ssize_t n)
{
    return call_for<2>(5, n, [&](at::Tensor* out) {
        const int64_t N = integer(a[1]), K = integer(a[2]);
        const rtn_code_format fmt = (rtn_code_format)integer(a[3]);
        const void* w = codes(a[0], N, K, fmt, "w_codes");
        const at::Tensor& like = tensor(a[0], "w_codes");
        const size_t b = rtn_linear_prepared_bytes(N, K), bt = truth(a[4]) ? rtn_linear_prepared_bytes(K, N) : 0;
        out[0] = make_bytes(b, like);
        if (bt) out[1] = make_bytes(bt, like);
        void *p = out[0].data_ptr(), *pt = bt ? out[1].data_ptr() : nullptr, *st = stream();
        const Unlocked u;
        return rtn_linear_prepare(fmt, w, N, K, p, b, pt, bt, st);
    });
}

// x, prepared, N, alpha_w, bias, act, residual, y_out, z_ckpt, workspace
PyObject* linear(PyObject*, Args a, Py_ssize_t n)
{
    return call_for<1>(10, n, [&](at::Tensor* out) {
        const at::Tensor& xt = matrix(a[0], "x");
        const c10::ScalarType type = xt.scalar_type();
        const rtn_dtype dt = dtype(type, "x");
        const int64_t M = xt.size(0), K = xt.size(1), N = integer(a[2]);
        int64_t ldx, ldr, ldy;
        const void* x = rows2d(xt, type, M, K, "x", ldx);
        const void* w = bytes_of(a[1], rtn_linear_prepared_bytes(N, K), "prepared");
        const AlphaN al(a[3], N);
        const void* bias = vector_of(a[4], type, N, "bias");
        const rtn_act act = (rtn_act)integer(a[5]);
        const void* res = rows2d(a[6], type, M, N, "residual", ldr);
        out[0] = given_or(a[7], "y_out", [&] { return make_rows(M, N, type, xt); });
        void* y = rows2d(out[0], type, M, N, "y_out", ldy);
        void* z = bytes_of(a[8], rtn_checkpoint_bytes(M, N), "z_ckpt");
        const size_t zb = raw_bytes(a[8], "z_ckpt"), need = rtn_linear_workspace_bytes(x, ldx, M, N, K, z != nullptr);
        at::Tensor work;
        if (need) work = given_or(a[9], "workspace", [&] { return make_bytes(need, xt); });
        void *ws = need ? scratch(work) : nullptr, *st = stream();
        const size_t wsb = need ? work.nbytes() : 0;
        const Unlocked u;
        return rtn_linear(dt, x, ldx, w, M, N, K, al.ptr, al.gran, bias, act, res, ldr, y, ldy, z, zb, ws, wsb, st);
    });
}

// x, ckpt
PyObject* checkpoint_pack(PyObject*, Args a, Py_ssize_t n)
{
    return call_for<1>(2, n, [&](at::Tensor* out) {
        const at::Tensor& t = matrix(a[0], "x");
        const rtn_dtype dt = dtype(t.scalar_type(), "x");
        const int64_t M = t.size(0), C = t.size(1);
        int64_t ld;
        const void* x = rows2d(t, t.scalar_type(), M, C, "x", ld);
        const size_t need = rtn_checkpoint_bytes(M, C);
        out[0] = given_or(a[1], "ckpt", [&] { return make_bytes(need, t); });
        void *k = bytes_of(out[0], need, "ckpt"), *st = stream();
        const size_t kb = out[0].nbytes();
        const Unlocked u;
        return rtn_checkpoint_pack(dt, x, ld, M, C, k, kb, st);
    });
}

// ckpt, M, C, float16 (else bfloat16), out
PyObject* checkpoint_unpack(PyObject*, Args a, Py_ssize_t n)
{
    return call_for<1>(5, n, [&](at::Tensor* out) {
        const at::Tensor& k = tensor(a[0], "ckpt");
        const int64_t M = integer(a[1]), C = integer(a[2]);
        const c10::ScalarType type = truth(a[3]) ? c10::kHalf : c10::kBFloat16;
        const void* kp = bytes_of(k, rtn_checkpoint_bytes(M, C), "ckpt");
        out[0] = given_or(a[4], "out", [&] { return make_rows(M, C, type, k); });
        int64_t ld;
        void* y = rows2d(out[0], type, M, C, "out", ld);
        const size_t kb = k.nbytes();
        const rtn_dtype dt = dtype(type, "out");
        void* st = stream();
        const Unlocked u;
        return rtn_checkpoint_unpack(dt, kp, kb, M, C, y, ld, st);
    });
}

// dy, prepared_t, K, alpha_w, x_ckpt, act, z_ckpt, want_dx, want_dw, want_dbias, dw in fp32, dx, dw, dbias, workspace
PyObject* linear_backward(PyObject*, Args a, Py_ssize_t n)
{
    return call_for<3>(15, n, [&](at::Tensor* out) {
        const at::Tensor& t = matrix(a[0], "dy");
        const c10::ScalarType type = t.scalar_type();
        const rtn_dtype dt = dtype(type, "dy");
        const int64_t M = t.size(0), N = t.size(1), K = integer(a[2]);
        int64_t lddy, lddx = K, lddw;
        const void* dy = rows2d(t, type, M, N, "dy", lddy);
        const void* w = bytes_of(a[1], rtn_linear_prepared_bytes(K, N), "prepared_t");
        const AlphaN al(a[3], N);
        const void* x = bytes_of(a[4], rtn_checkpoint_bytes(M, K), "x_ckpt");
        const rtn_act act = (rtn_act)integer(a[5]);
        const void* z = bytes_of(a[6], rtn_checkpoint_bytes(M, N), "z_ckpt");
        const size_t xb = raw_bytes(a[4], "x_ckpt"), zb = raw_bytes(a[6], "z_ckpt");
        void *dx = nullptr, *dw = nullptr, *db = nullptr;
        rtn_dtype dwt = dt;
        if (truth(a[7])) {
            out[0] = given_or(a[11], "dx", [&] { return make_rows(M, K, type, t); });
            dx = rows2d(out[0], type, M, K, "dx", lddx);
        }
        if (truth(a[8])) {
            out[1] = given_or(a[12], "dw", [&] { return make_rows(N, K, truth(a[10]) ? c10::kFloat : type, t); });
            dwt = dtype(out[1].scalar_type(), "dw", true);
            dw = rows2d(out[1], out[1].scalar_type(), N, K, "dw", lddw);
            if (lddw != K) fail(PyExc_AssertionError, "%s: a contiguous tensor is required", "dw");
        }
        if (truth(a[9])) {
            out[2] = given_or(a[13], "dbias", [&] { return at::empty({N}, t.options()); });
            if (!out[2].is_cuda() || out[2].scalar_type() != type || !out[2].is_contiguous() || out[2].numel() != N)
                fail(PyExc_AssertionError, "%s: a contiguous device tensor of dy's type, one entry per output, is required", "dbias");
            db = out[2].data_ptr();
        }
        const at::Tensor work = given_or(a[14], "workspace", [&] { return make_bytes(rtn_linear_backward_workspace_bytes(M, N, K), t); });
        void *ws = scratch(work), *st = stream();
        const size_t wsb = work.nbytes();
        const Unlocked u;
        return rtn_linear_backward(dt, dy, lddy, x, xb, z, zb, act, w, M, N, K, al.ptr, al.gran, dx, lddx, dw, dwt, db, ws, wsb, st);
    });
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(pack), FAST(gemm), FAST(conv2d), FAST(conv2d_ternarize), FAST(depthwise), FAST(weight_gemm),
                         FAST(weight_conv2d_prepared), FAST(activation_backward), FAST(weight_backward),
                         FAST(linear_prepare), FAST(linear), FAST(checkpoint_pack), FAST(checkpoint_unpack), FAST(linear_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
