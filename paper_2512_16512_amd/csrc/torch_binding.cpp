// The common calls of matmul(), conv2d_nchw() and the norm, 8-bit and grouped
// operators over torch tensors, without the Python interpreter in between: a
// product of a few microseconds on the GPU waited for its caller, which spent 10 us in
// argument checks (2.3), torch.empty (1.7), the stream lookup (1.9) and ctypes
// around 3.3 us of launch; through this module it is 4.2 us.
//
// The functions return the output tensor (or tensors), or None for every call that is
// not the plain one (a tensor subclass, a transform or a dispatch mode is
// active, an operand of another device, type, shape or layout, an error
// status): the caller then takes the Python path, which checks and reports.
// Nothing is kept from one call to the next.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/xtc.h"

namespace {

// A plain strided tensor in GPU memory: an instance of torch.Tensor itself
// (or a Parameter) with no other dispatch key than the dense GPU backend's
// and autograd's.
bool plain(PyObject *o, const at::Tensor **out) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage()) return false;
    const c10::DispatchKeySet usual({c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA,
                                     c10::DispatchKey::ADInplaceOrView, c10::DispatchKey::AutocastCUDA});
    if (t.key_set().raw_repr() & ~usual.raw_repr()) return false;
    *out = &t;
    return true;
}

bool modes_active() {
    return c10::impl::TorchDispatchModeTLS::any_modes_set() ||
           at::impl::PythonTorchFunctionTLS::stack_len() > 0 ||
           (c10::impl::tls_local_dispatch_key_set().included_.raw_repr() &
            ~c10::DispatchKeySet({c10::DispatchKey::BackendSelect, c10::DispatchKey::ADInplaceOrView}).raw_repr());
}

bool dtype_code(const at::Tensor &t, xtc_dtype *code) {
    if (t.scalar_type() == at::kFloat) *code = XTC_F32;
    else if (t.scalar_type() == at::kBFloat16) *code = XTC_BF16;
    else return false;
    return true;
}

bool row_major(const at::Tensor &t) { return t.dim() == 2 && (t.size(1) <= 1 || t.stride(1) == 1); }

void *stream_of(const at::Tensor &t) {
    return static_cast<void *>(c10::hip::getCurrentHIPStream(t.device().index()).stream());
}

// matmul(a, b, out or None, relu)
PyObject *matmul(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *a, *b, *c = nullptr;
    xtc_dtype dt, dtb;
    if (n != 4 || modes_active() || !plain(args[0], &a) || !plain(args[1], &b) ||
        (args[2] != Py_None && !plain(args[2], &c)) || (args[3] != Py_True && args[3] != Py_False))
        Py_RETURN_NONE;
    if (!row_major(*a) || !row_major(*b) || !dtype_code(*a, &dt) || !dtype_code(*b, &dtb) || dt != dtb ||
        a->device() != b->device() || a->size(1) != b->size(0))
        Py_RETURN_NONE;
    const int64_t M = a->size(0), K = a->size(1), N = b->size(1);
    if (c && (!row_major(*c) || c->scalar_type() != at::kFloat || c->device() != a->device() ||
              c->size(0) != M || c->size(1) != N))
        Py_RETURN_NONE;
    try {
        at::Tensor fresh;
        if (!c) {
            fresh = at::empty({M, N}, at::TensorOptions().dtype(at::kFloat).device(a->device()));
            c = &fresh;
        }
        const int64_t lda = M > 1 ? a->stride(0) : (K > 1 ? K : 1), ldb = K > 1 ? b->stride(0) : (N > 1 ? N : 1),
                      ldc = M > 1 ? c->stride(0) : (N > 1 ? N : 1);
        const void *pa = a->data_ptr(), *pb = b->data_ptr();
        float *pc = static_cast<float *>(c->data_ptr());
        void *stream = stream_of(*a);
        xtc_status st;
        Py_BEGIN_ALLOW_THREADS
        st = (args[3] == Py_True ? xtc_matmul_relu : xtc_matmul)(M, N, K, pa, lda, pb, ldb, pc, ldc, dt, nullptr,
                                                                 stream);
        Py_END_ALLOW_THREADS
        if (st != XTC_OK) Py_RETURN_NONE;
        if (args[2] != Py_None) return Py_NewRef(args[2]);
        return THPVariable_Wrap(std::move(fresh));
    } catch (...) {
        Py_RETURN_NONE;   // the Python path meets the same error and reports it
    }
}

// An int, or a tuple of two ints.
bool pair_of(PyObject *o, int64_t *h, int64_t *w) {
    auto value = [](PyObject *v, int64_t *out) {
        if (!PyLong_CheckExact(v)) return false;
        int overflow = 0;
        *out = PyLong_AsLongLongAndOverflow(v, &overflow);
        return overflow == 0;
    };
    if (PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 2)
        return value(PyTuple_GET_ITEM(o, 0), h) && value(PyTuple_GET_ITEM(o, 1), w);
    if (!value(o, h)) return false;
    *w = *h;
    return true;
}

// conv2d_nchw(x, w, stride, pad, out or None, relu)
PyObject *conv2d_nchw(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *x, *w, *y = nullptr;
    xtc_dtype dt, dtw;
    int64_t sh, sw, ph, pw;
    if (n != 6 || modes_active() || !plain(args[0], &x) || !plain(args[1], &w) || !pair_of(args[2], &sh, &sw) ||
        !pair_of(args[3], &ph, &pw) || (args[4] != Py_None && !plain(args[4], &y)) ||
        (args[5] != Py_True && args[5] != Py_False))
        Py_RETURN_NONE;
    if (x->dim() != 4 || w->dim() != 4 || !x->is_contiguous() || !w->is_contiguous() || !dtype_code(*x, &dt) ||
        !dtype_code(*w, &dtw) || dt != dtw || x->device() != w->device() || x->size(1) != w->size(1))
        Py_RETURN_NONE;
    const int64_t N = x->size(0), C = x->size(1), H = x->size(2), W = x->size(3), OC = w->size(0), R = w->size(2),
                  S = w->size(3);
    constexpr int64_t kLimit = int64_t(1) << 30;   // (also keeps the sums below inside 64 bits)
    if (sh < 1 || sw < 1 || ph < 0 || pw < 0 || sh > kLimit || sw > kLimit || ph > kLimit || pw > kLimit)
        Py_RETURN_NONE;
    if (R < 1 || S < 1 || H + 2 * ph < R || W + 2 * pw < S) Py_RETURN_NONE;
    const int64_t OH = (H + 2 * ph - R) / sh + 1, OW = (W + 2 * pw - S) / sw + 1;
    if (y && (y->dim() != 4 || !y->is_contiguous() || y->scalar_type() != at::kFloat || y->device() != x->device() ||
              y->size(0) != N || y->size(1) != OC || y->size(2) != OH || y->size(3) != OW))
        Py_RETURN_NONE;
    try {
        at::Tensor fresh;
        if (!y) {
            fresh = at::empty({N, OC, OH, OW}, at::TensorOptions().dtype(at::kFloat).device(x->device()));
            y = &fresh;
        }
        const void *px = x->data_ptr(), *pt = w->data_ptr();
        float *py = static_cast<float *>(y->data_ptr());
        void *stream = stream_of(*x);
        xtc_status st;
        Py_BEGIN_ALLOW_THREADS
        st = (args[5] == Py_True ? xtc_conv2d_nchw_relu : xtc_conv2d_nchw)(N, C, H, W, OC, R, S, sh, sw, ph, pw, px,
                                                                           pt, py, dt, nullptr, stream);
        Py_END_ALLOW_THREADS
        if (st != XTC_OK) Py_RETURN_NONE;
        if (args[4] != Py_None) return Py_NewRef(args[4]);
        return THPVariable_Wrap(std::move(fresh));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// ------------------------------------- norms, 8-bit and grouped products

constexpr at::ScalarType kE4m3 = at::kFloat8_e4m3fn;
int64_t blocks_of(int64_t n) { return (n + 127) / 128; }
int64_t at_least_1(int64_t n) { return n > 1 ? n : 1; }
// Row stride of a matrix (the last two axes), its length where there is one row.
int64_t row_stride(const at::Tensor &t) {
    const int64_t d = t.dim();
    return t.size(d - 2) > 1 ? t.stride(d - 2) : at_least_1(t.size(d - 1));
}
int64_t family_stride(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : 0; }
bool unit(const at::Tensor &t) { return t.size(t.dim() - 1) <= 1 || t.stride(t.dim() - 1) == 1; }

bool matrix(const at::Tensor &t, at::ScalarType type, int64_t rows, int64_t cols, const at::Tensor &like) {
    return t.dim() == 2 && t.scalar_type() == type && t.size(0) == rows && t.size(1) == cols && unit(t) &&
           t.device() == like.device();
}
bool family(const at::Tensor &t, at::ScalarType type, int64_t n, int64_t rows, int64_t cols, const at::Tensor &like) {
    return t.dim() == 3 && t.scalar_type() == type && t.size(0) == n && t.size(1) == rows && t.size(2) == cols &&
           unit(t) && t.device() == like.device();
}
bool vector_of(const at::Tensor &t, at::ScalarType type, int64_t n, const at::Tensor &like) {
    return t.dim() == 1 && t.scalar_type() == type && t.size(0) == n && t.is_contiguous() && t.device() == like.device();
}
// The arguments at..at + N - 1 as plain tensors (null where None is allowed by `maybe`).
template <int N>
bool tensors(PyObject *const *args, const at::Tensor *(&out)[N], unsigned maybe = 0) {
    for (int i = 0; i < N; ++i) {
        out[i] = nullptr;
        if ((maybe >> i & 1) && args[i] == Py_None) continue;
        if (!plain(args[i], &out[i])) return false;
    }
    return true;
}
bool truth(PyObject *o) { return o == Py_True || o == Py_False; }
const void *data(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }

// (Straight from the GPU's allocator: the dispatcher in front of at::empty costs as
// much again, and a norm makes four tensors.)
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const at::Tensor &like) {
    return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
}

// The output of a product: `given`, or a new one of the type code in `o` (0
// fp32, 1 bf16).
bool result(const at::Tensor *given, PyObject *o, at::IntArrayRef shape, const at::Tensor &like, at::Tensor *out,
            xtc_dtype *code) {
    if (given) {
        if (o != Py_None || !dtype_code(*given, code) || given->sizes() != shape || !unit(*given) ||
            given->device() != like.device())
            return false;
        *out = *given;
        return true;
    }
    if (o == Py_None) {
        *code = XTC_F32;
    } else {
        if (!THPDtype_Check(o)) return false;
        const at::ScalarType t = reinterpret_cast<THPDtype *>(o)->scalar_type;
        if (t != at::kFloat && t != at::kBFloat16) return false;
        *code = t == at::kFloat ? XTC_F32 : XTC_BF16;
    }
    *out = fresh(shape, *code == XTC_F32 ? at::kFloat : at::kBFloat16, like);
    return true;
}

// f(args...) without the interpreter's lock; the arguments are evaluated before.
template <typename... P, typename... A>
xtc_status unlocked(xtc_status (*f)(P...), A... args) {
    xtc_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f(args...);
    Py_END_ALLOW_THREADS
    return st;
}

PyObject *wrapped(at::Tensor t) { return t.defined() ? THPVariable_Wrap(std::move(t)) : Py_NewRef(Py_None); }

// rmsnorm(x, weight, residual or None, eps, quantize): (out, scale or None, residual, rstd)
PyObject *rmsnorm(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[3];
    xtc_dtype dt, dtw;
    if (n != 5 || modes_active() || !tensors(args, t, 4) || !PyFloat_CheckExact(args[3]) || !truth(args[4])) Py_RETURN_NONE;
    const at::Tensor &x = *t[0], &w = *t[1];
    if (!row_major(x) || !dtype_code(x, &dt)) Py_RETURN_NONE;
    const int64_t T = x.size(0), D = x.size(1);
    // (of no columns the library's call writes nothing, but there is an rstd to fill)
    if (D == 0 || !dtype_code(w, &dtw) || (dtw != dt && dtw != XTC_F32) || !vector_of(w, w.scalar_type(), D, x) ||
        (t[2] && !matrix(*t[2], x.scalar_type(), T, D, x)))
        Py_RETURN_NONE;
    try {
        const bool quantize = args[4] == Py_True;
        at::Tensor out = fresh({T, D}, quantize ? kE4m3 : x.scalar_type(), x), scale, total, rstd = fresh({T}, at::kFloat, x);
        if (quantize) scale = fresh({T, blocks_of(D)}, at::kFloat, x);
        if (t[2]) total = fresh({T, D}, x.scalar_type(), x);
        const float eps = (float)PyFloat_AS_DOUBLE(args[3]);
        float *ps = quantize ? static_cast<float *>(scale.data_ptr()) : nullptr;
        void *ph = t[2] ? total.data_ptr() : nullptr;
        const int64_t ldr = t[2] ? row_stride(*t[2]) : 0;
        void *stream = stream_of(x);
        if (unlocked(xtc_rmsnorm, T, D, x.data_ptr(), row_stride(x), data(t[2]), ldr, w.data_ptr(), eps,
                     out.data_ptr(), at_least_1(D), ps, blocks_of(D), ph, D, static_cast<float *>(rstd.data_ptr()), dt, dtw,
                     quantize ? XTC_FP8 : dt, stream) != XTC_OK)
            Py_RETURN_NONE;
        PyObject *r = PyTuple_New(4);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, wrapped(std::move(out)));
        PyTuple_SET_ITEM(r, 1, wrapped(std::move(scale)));
        PyTuple_SET_ITEM(r, 2, t[2] ? wrapped(std::move(total)) : Py_NewRef(args[0]));
        PyTuple_SET_ITEM(r, 3, wrapped(std::move(rstd)));
        return r;
    } catch (...) {
        Py_RETURN_NONE;
    }
}

PyObject *pair(at::Tensor a, at::Tensor b) {
    PyObject *r = PyTuple_New(2);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, wrapped(std::move(a)));
    PyTuple_SET_ITEM(r, 1, wrapped(std::move(b)));
    return r;
}

// rmsnorm_backward(dy, x, weight, rstd, dresidual or None): (dx, dweight)
PyObject *rmsnorm_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[5];
    xtc_dtype dt, dtw;
    if (n != 5 || modes_active() || !tensors(args, t, 16)) Py_RETURN_NONE;
    const at::Tensor &dy = *t[0], &x = *t[1], &w = *t[2], &rstd = *t[3];
    if (!row_major(x) || !dtype_code(x, &dt)) Py_RETURN_NONE;
    const int64_t T = x.size(0), D = x.size(1);
    if (!matrix(dy, x.scalar_type(), T, D, x) || !dtype_code(w, &dtw) || (dtw != dt && dtw != XTC_F32) ||
        !vector_of(w, w.scalar_type(), D, x) || !vector_of(rstd, at::kFloat, T, x) ||
        (t[4] && !matrix(*t[4], x.scalar_type(), T, D, x)))
        Py_RETURN_NONE;
    try {
        const int64_t size = xtc_rmsnorm_backward_workspace(T, D);
        if (size < 0) Py_RETURN_NONE;
        at::Tensor dx = fresh({T, D}, x.scalar_type(), x), dw = fresh({D}, at::kFloat, x), work = fresh({size}, at::kByte, x);
        const int64_t lddr = t[4] ? row_stride(*t[4]) : 0;
        void *stream = stream_of(x);
        if (unlocked(xtc_rmsnorm_backward, T, D, dy.data_ptr(), row_stride(dy), x.data_ptr(), row_stride(x),
                     w.data_ptr(), static_cast<const float *>(rstd.data_ptr()), data(t[4]), lddr, dx.data_ptr(), at_least_1(D),
                     static_cast<float *>(dw.data_ptr()), work.data_ptr(), size, dt, dtw, stream) != XTC_OK)
            Py_RETURN_NONE;
        return pair(std::move(dx), std::move(dw));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// The tensors as a tuple (None for undefined ones).
template <int N>
PyObject *tuple_of(at::Tensor (&t)[N]) {
    PyObject *r = PyTuple_New(N);
    if (!r) return nullptr;
    for (int i = 0; i < N; ++i) PyTuple_SET_ITEM(r, i, wrapped(std::move(t[i])));
    return r;
}

// layernorm(x, weight, bias or None, residual or None, eps, quantize): (out, scale or None, residual, mean, rstd)
PyObject *layernorm(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[4];
    xtc_dtype dt, dtw;
    if (n != 6 || modes_active() || !tensors(args, t, 4 | 8) || !PyFloat_CheckExact(args[4]) || !truth(args[5])) Py_RETURN_NONE;
    const at::Tensor &x = *t[0], &w = *t[1];
    if (!row_major(x) || !dtype_code(x, &dt)) Py_RETURN_NONE;
    const int64_t T = x.size(0), D = x.size(1);
    // (of no columns the library's call writes nothing, but there are a mean and an rstd to fill)
    if (D == 0 || !dtype_code(w, &dtw) || (dtw != dt && dtw != XTC_F32) || !vector_of(w, w.scalar_type(), D, x) ||
        (t[2] && !vector_of(*t[2], w.scalar_type(), D, x)) || (t[3] && !matrix(*t[3], x.scalar_type(), T, D, x)))
        Py_RETURN_NONE;
    try {
        const c10::DeviceGuard on(x.device());
        const bool quantize = args[5] == Py_True;
        at::Tensor r[5];     // out, scale, residual, mean, rstd
        r[0] = fresh({T, D}, quantize ? kE4m3 : x.scalar_type(), x);
        if (quantize) r[1] = fresh({T, blocks_of(D)}, at::kFloat, x);
        r[2] = t[3] ? fresh({T, D}, x.scalar_type(), x) : x;
        r[3] = fresh({T}, at::kFloat, x);
        r[4] = fresh({T}, at::kFloat, x);
        const float eps = (float)PyFloat_AS_DOUBLE(args[4]);
        float *ps = quantize ? static_cast<float *>(r[1].data_ptr()) : nullptr;
        void *ph = t[3] ? r[2].data_ptr() : nullptr;
        const int64_t ldr = t[3] ? row_stride(*t[3]) : 0;
        void *stream = stream_of(x);
        if (unlocked(xtc_layernorm, T, D, x.data_ptr(), row_stride(x), data(t[3]), ldr, w.data_ptr(), data(t[2]), eps,
                     r[0].data_ptr(), D, ps, blocks_of(D), ph, D, static_cast<float *>(r[3].data_ptr()),
                     static_cast<float *>(r[4].data_ptr()), dt, dtw, quantize ? XTC_FP8 : dt, stream) != XTC_OK)
            Py_RETURN_NONE;
        return tuple_of(r);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// layernorm_backward(dy, x, weight, mean, rstd, dresidual or None): (dx, dweight, dbias)
PyObject *layernorm_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[6];
    xtc_dtype dt, dtw;
    if (n != 6 || modes_active() || !tensors(args, t, 32)) Py_RETURN_NONE;
    const at::Tensor &dy = *t[0], &x = *t[1], &w = *t[2], &mean = *t[3], &rstd = *t[4];
    if (!row_major(x) || !dtype_code(x, &dt)) Py_RETURN_NONE;
    const int64_t T = x.size(0), D = x.size(1);
    if (!matrix(dy, x.scalar_type(), T, D, x) || !dtype_code(w, &dtw) || (dtw != dt && dtw != XTC_F32) ||
        !vector_of(w, w.scalar_type(), D, x) || !vector_of(mean, at::kFloat, T, x) || !vector_of(rstd, at::kFloat, T, x) ||
        (t[5] && !matrix(*t[5], x.scalar_type(), T, D, x)))
        Py_RETURN_NONE;
    try {
        const c10::DeviceGuard on(x.device());
        const int64_t size = xtc_layernorm_backward_workspace(T, D);
        if (size < 0) Py_RETURN_NONE;
        at::Tensor r[3] = {fresh({T, D}, x.scalar_type(), x), fresh({D}, at::kFloat, x), fresh({D}, at::kFloat, x)};
        at::Tensor work = fresh({size}, at::kByte, x);
        const int64_t lddr = t[5] ? row_stride(*t[5]) : 0;
        void *stream = stream_of(x);
        if (unlocked(xtc_layernorm_backward, T, D, dy.data_ptr(), row_stride(dy), x.data_ptr(), row_stride(x),
                     w.data_ptr(), static_cast<const float *>(mean.data_ptr()), static_cast<const float *>(rstd.data_ptr()),
                     data(t[5]), lddr, r[0].data_ptr(), at_least_1(D), static_cast<float *>(r[1].data_ptr()),
                     static_cast<float *>(r[2].data_ptr()), work.data_ptr(), size, dt, dtw, stream) != XTC_OK)
            Py_RETURN_NONE;
        return tuple_of(r);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// quantize_fp8(x, block_rows): (q, scale)
PyObject *quantize_fp8(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *x;
    xtc_dtype dt;
    if (n != 2 || modes_active() || !plain(args[0], &x) || !PyLong_CheckExact(args[1]) || !row_major(*x) ||
        !dtype_code(*x, &dt))
        Py_RETURN_NONE;
    int overflow = 0;
    const long rows = PyLong_AsLongAndOverflow(args[1], &overflow);
    if (overflow || (rows != 1 && rows != 128)) Py_RETURN_NONE;
    const int64_t M = x->size(0), K = x->size(1);
    try {
        at::Tensor q = fresh({M, K}, kE4m3, *x), s = fresh({rows == 1 ? M : blocks_of(M), blocks_of(K)}, at::kFloat, *x);
        void *stream = stream_of(*x);
        if (unlocked(xtc_quantize_fp8, M, K, x->data_ptr(), row_stride(*x), rows, q.data_ptr(), at_least_1(K),
                     static_cast<float *>(s.data_ptr()), blocks_of(K), dt, stream) != XTC_OK)
            Py_RETURN_NONE;
        return pair(std::move(q), std::move(s));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// matmul_fp8(a, a_scale, b, b_scale, out or None, relu, dtype or None)
PyObject *matmul_fp8(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[5];
    if (n != 7 || modes_active() || !tensors(args, t, 16) || !truth(args[5])) Py_RETURN_NONE;
    const at::Tensor &a = *t[0], &sa = *t[1], &b = *t[2], &sb = *t[3];
    if (a.dim() != 2 || b.dim() != 2) Py_RETURN_NONE;
    const int64_t M = a.size(0), K = a.size(1), N = b.size(0), kb = blocks_of(K);
    if (!matrix(a, kE4m3, M, K, a) || !matrix(b, kE4m3, N, K, a) || !matrix(sa, at::kFloat, M, kb, a) ||
        !matrix(sb, at::kFloat, blocks_of(N), kb, a))
        Py_RETURN_NONE;
    try {
        at::Tensor c;
        xtc_dtype code;
        if (!result(t[4], args[6], {M, N}, a, &c, &code)) Py_RETURN_NONE;
        void *stream = stream_of(a);
        if (unlocked(xtc_matmul_fp8, M, N, K, a.data_ptr(), row_stride(a), static_cast<const float
                     *>(sa.data_ptr()), row_stride(sa), b.data_ptr(), row_stride(b), static_cast<const float *>(sb.data_ptr()),
                     row_stride(sb), c.data_ptr(), row_stride(c), code, args[5] == Py_True, stream) != XTC_OK)
            Py_RETURN_NONE;
        return t[4] ? Py_NewRef(args[4]) : wrapped(std::move(c));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

xtc_dtype code_of(const at::Tensor *t) { return !t || t->scalar_type() == at::kFloat ? XTC_F32 : XTC_BF16; }
bool either(const at::Tensor &t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
bool small_int(PyObject *o, long *out) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    *out = PyLong_AsLongAndOverflow(o, &overflow);
    return overflow == 0 && *out > -(1L << 30) && *out < (1L << 30);
}

// linear(a, b, bias or None, residual or None, activation's code, transpose_b, keep, out or None, dtype or None): out,
// or (out, z)
PyObject *linear(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[4], *given = nullptr;
    long act;
    if (n != 9 || modes_active() || !tensors(args, t, 4 | 8) || !small_int(args[4], &act) || !truth(args[5]) ||
        !truth(args[6]) || (args[7] != Py_None && !plain(args[7], &given)))
        Py_RETURN_NONE;
    const at::Tensor &a = *t[0], &b = *t[1];
    if (a.dim() != 2 || b.dim() != 2) Py_RETURN_NONE;
    const bool turned = args[5] == Py_True, keep = args[6] == Py_True;
    const int64_t T = a.size(0), K = a.size(1), N = b.size(turned ? 0 : 1);
    if (!matrix(a, at::kBFloat16, T, K, a) || !matrix(b, at::kBFloat16, turned ? N : K, turned ? K : N, a) ||
        (t[2] && (!either(*t[2]) || !vector_of(*t[2], t[2]->scalar_type(), N, a))) ||
        (t[3] && (!either(*t[3]) || !matrix(*t[3], t[3]->scalar_type(), T, N, a))))
        Py_RETURN_NONE;
    try {
        const c10::DeviceGuard on(a.device());
        at::Tensor r[2], work;
        xtc_dtype code;
        if (!result(given, args[8], {T, N}, a, &r[0], &code)) Py_RETURN_NONE;
        if (keep) r[1] = fresh({T, N}, r[0].scalar_type(), a);
        const int64_t size = xtc_linear_workspace(T, N, K, a.data_ptr(), row_stride(a), b.data_ptr(), row_stride(b), turned);
        if (size < 0) Py_RETURN_NONE;
        if (size > 0) work = fresh({size}, at::kByte, a);
        void *stream = stream_of(a);
        if (unlocked(xtc_linear, T, N, K, a.data_ptr(), row_stride(a), b.data_ptr(), row_stride(b), turned, data(t[2]),
                     code_of(t[2]), data(t[3]), t[3] ? row_stride(*t[3]) : 0, code_of(t[3]), (int32_t)act,
                     r[0].data_ptr(), row_stride(r[0]), keep ? r[1].data_ptr() : nullptr, at_least_1(N),
                     size > 0 ? work.data_ptr() : nullptr, size, XTC_BF16, code, stream) != XTC_OK)
            Py_RETURN_NONE;
        if (keep) return tuple_of(r);
        return given ? Py_NewRef(args[7]) : wrapped(std::move(r[0]));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// linear_wgrad(a, dy, out or None, dtype or None)
PyObject *linear_wgrad(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[3];
    if (n != 4 || modes_active() || !tensors(args, t, 4)) Py_RETURN_NONE;
    const at::Tensor &a = *t[0], &dy = *t[1];
    if (a.dim() != 2 || dy.dim() != 2) Py_RETURN_NONE;
    const int64_t T = a.size(0), K = a.size(1), N = dy.size(1);
    if (!matrix(a, at::kBFloat16, T, K, a) || !matrix(dy, at::kBFloat16, T, N, a)) Py_RETURN_NONE;
    try {
        const c10::DeviceGuard on(a.device());
        at::Tensor c, work;
        xtc_dtype code;
        if (!result(t[2], args[3], {K, N}, a, &c, &code)) Py_RETURN_NONE;
        const int64_t size = xtc_linear_wgrad_workspace(T, N, K, a.data_ptr(), row_stride(a), dy.data_ptr(), row_stride(dy));
        if (size < 0) Py_RETURN_NONE;
        if (size > 0) work = fresh({size}, at::kByte, a);
        void *stream = stream_of(a);
        if (unlocked(xtc_linear_wgrad, T, N, K, a.data_ptr(), row_stride(a), dy.data_ptr(), row_stride(dy), c.data_ptr(),
                     row_stride(c), size > 0 ? work.data_ptr() : nullptr, size, XTC_BF16, code, stream) != XTC_OK)
            Py_RETURN_NONE;
        return t[2] ? Py_NewRef(args[2]) : wrapped(std::move(c));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// activation_backward(dy, z, activation's code): (dz, dbias)
PyObject *activation_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[2];
    long act;
    if (n != 3 || modes_active() || !tensors(args, t) || !small_int(args[2], &act)) Py_RETURN_NONE;
    const at::Tensor &dy = *t[0], &z = *t[1];
    if (dy.dim() != 2 || !either(dy) || !either(z)) Py_RETURN_NONE;
    const int64_t T = dy.size(0), N = dy.size(1);
    if (!matrix(dy, dy.scalar_type(), T, N, dy) || !matrix(z, z.scalar_type(), T, N, dy)) Py_RETURN_NONE;
    try {
        const c10::DeviceGuard on(dy.device());
        const int64_t size = xtc_activation_backward_workspace(T, N);
        if (size < 0) Py_RETURN_NONE;
        at::Tensor dz = fresh({T, N}, at::kBFloat16, dy), db = fresh({N}, at::kFloat, dy), work = fresh({size}, at::kByte, dy);
        void *stream = stream_of(dy);
        if (unlocked(xtc_activation_backward, T, N, dy.data_ptr(), row_stride(dy), code_of(&dy), z.data_ptr(),
                     row_stride(z), code_of(&z), (int32_t)act, dz.data_ptr(), at_least_1(N),
                     static_cast<float *>(db.data_ptr()), work.data_ptr(), size, stream) != XTC_OK)
            Py_RETURN_NONE;
        return pair(std::move(dz), std::move(db));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// matmul_grouped(a, b, ends, transpose_b, out or None, relu, dtype or None)
PyObject *matmul_grouped(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[3], *given = nullptr;
    if (n != 7 || modes_active() || !tensors(args, t) || !truth(args[3]) || !truth(args[5]) ||
        (args[4] != Py_None && !plain(args[4], &given)))
        Py_RETURN_NONE;
    const at::Tensor &a = *t[0], &b = *t[1], &ends = *t[2];
    if (a.dim() != 2 || b.dim() != 3) Py_RETURN_NONE;
    const bool turned = args[3] == Py_True;
    const int64_t T = a.size(0), K = a.size(1), G = b.size(0), N = b.size(turned ? 1 : 2);
    if (!matrix(a, at::kBFloat16, T, K, a) || !family(b, at::kBFloat16, G, turned ? N : K, turned ? K : N, a) ||
        !vector_of(ends, at::kInt, G, a))
        Py_RETURN_NONE;
    try {
        at::Tensor c;
        xtc_dtype code;
        if (!result(given, args[6], {T, N}, a, &c, &code)) Py_RETURN_NONE;
        void *stream = stream_of(a);
        if (unlocked(xtc_matmul_grouped, G, T, N, K, a.data_ptr(), row_stride(a), b.data_ptr(), row_stride(b),
                     family_stride(b), turned, static_cast<const int32_t *>(ends.data_ptr()), c.data_ptr(), row_stride(c),
                     XTC_BF16, code, args[5] == Py_True, stream) != XTC_OK)
            Py_RETURN_NONE;
        return given ? Py_NewRef(args[4]) : wrapped(std::move(c));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// matmul_grouped_wgrad(a, dy, ends, out or None, dtype or None)
PyObject *matmul_grouped_wgrad(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[4];
    if (n != 5 || modes_active() || !tensors(args, t, 8)) Py_RETURN_NONE;
    const at::Tensor &a = *t[0], &dy = *t[1], &ends = *t[2];
    if (a.dim() != 2 || dy.dim() != 2 || ends.dim() != 1) Py_RETURN_NONE;
    const int64_t T = a.size(0), K = a.size(1), N = dy.size(1), G = ends.size(0);
    if (!matrix(a, at::kBFloat16, T, K, a) || !matrix(dy, at::kBFloat16, T, N, a) || !vector_of(ends, at::kInt, G, a))
        Py_RETURN_NONE;
    try {
        at::Tensor c;
        xtc_dtype code;
        if (!result(t[3], args[4], {G, K, N}, a, &c, &code)) Py_RETURN_NONE;
        void *stream = stream_of(a);
        if (unlocked(xtc_matmul_grouped_wgrad, G, T, N, K, a.data_ptr(), row_stride(a), dy.data_ptr(),
                     row_stride(dy), static_cast<const int32_t *>(ends.data_ptr()), c.data_ptr(), row_stride(c),
                     family_stride(c), XTC_BF16, code, stream) != XTC_OK)
            Py_RETURN_NONE;
        return t[3] ? Py_NewRef(args[3]) : wrapped(std::move(c));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// matmul_grouped_fp8(a, a_scale, b, b_scale, ends, out or None, relu, dtype or None)
PyObject *matmul_grouped_fp8(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[6];
    if (n != 8 || modes_active() || !tensors(args, t, 32) || !truth(args[6])) Py_RETURN_NONE;
    const at::Tensor &a = *t[0], &sa = *t[1], &b = *t[2], &sb = *t[3], &ends = *t[4];
    if (a.dim() != 2 || b.dim() != 3) Py_RETURN_NONE;
    const int64_t T = a.size(0), K = a.size(1), G = b.size(0), N = b.size(1), kb = blocks_of(K);
    if (!matrix(a, kE4m3, T, K, a) || !family(b, kE4m3, G, N, K, a) || !matrix(sa, at::kFloat, T, kb, a) ||
        !family(sb, at::kFloat, G, blocks_of(N), kb, a) || !vector_of(ends, at::kInt, G, a))
        Py_RETURN_NONE;
    try {
        at::Tensor c;
        xtc_dtype code;
        if (!result(t[5], args[7], {T, N}, a, &c, &code)) Py_RETURN_NONE;
        void *stream = stream_of(a);
        if (unlocked(xtc_matmul_grouped_fp8, G, T, N, K, a.data_ptr(), row_stride(a), static_cast<const float
                     *>(sa.data_ptr()), row_stride(sa), b.data_ptr(), row_stride(b), family_stride(b), static_cast<const float
                     *>(sb.data_ptr()), row_stride(sb), family_stride(sb), static_cast<const int32_t *>(ends.data_ptr()),
                     c.data_ptr(), row_stride(c), code, args[6] == Py_True, stream) != XTC_OK)
            Py_RETURN_NONE;
        return t[5] ? Py_NewRef(args[5]) : wrapped(std::move(c));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

bool contiguous(const at::Tensor &t, at::ScalarType type, at::IntArrayRef shape, const at::Tensor &like) {
    return t.scalar_type() == type && t.sizes() == shape && t.is_contiguous() && t.device() == like.device();
}
template <typename T>
T *as(const at::Tensor &t) { return static_cast<T *>(t.data_ptr()); }
template <typename T>
T *as(const at::Tensor *t) { return t ? as<T>(*t) : nullptr; }

// route_experts(scores, top, mask or None): (expert, p, row, token, counts, ends, loss)
PyObject *route_experts(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *s, *mask = nullptr;
    xtc_dtype dt;
    long top;
    if (n != 3 || modes_active() || !plain(args[0], &s) || !small_int(args[1], &top) ||
        (args[2] != Py_None && !plain(args[2], &mask)) || !row_major(*s) || !dtype_code(*s, &dt))
        Py_RETURN_NONE;
    const int64_t T = s->size(0), E = s->size(1);
    if (top < 1 || top > E || (mask && !contiguous(*mask, at::kBool, {T}, *s))) Py_RETURN_NONE;
    try {
        const c10::DeviceGuard on(s->device());
        const int64_t size = xtc_route_experts_workspace(T, E);
        if (size < 0) Py_RETURN_NONE;
        // (one allocation for the results, each at a multiple of 64 bytes of it: eight cost more than the kernel)
        int64_t at = 0;
        auto place = [&](int64_t values) {
            const int64_t here = at;
            at += (values + 15) / 16 * 16;
            return here;
        };
        const int64_t n_all = T * top, o_e = place(n_all), o_p = place(n_all), o_r = place(n_all), o_t = place(n_all),
                      o_c = place(E), o_n = place(E), o_l = place(1);
        const at::Tensor all = fresh({at}, at::kInt, *s);
        auto part = [&](at::ScalarType type, at::IntArrayRef shape, int64_t offset) {
            at::Tensor v = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(),
                                                                    c10::scalarTypeToTypeMeta(type));
            v.unsafeGetTensorImpl()->set_storage_offset(offset);
            v.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
            return v;
        };
        at::Tensor r[7] = {part(at::kInt, {T, top}, o_e), part(at::kFloat, {T, top}, o_p), part(at::kInt, {T, top}, o_r),
                           part(at::kInt, {n_all}, o_t),  part(at::kInt, {E}, o_c),        part(at::kInt, {E}, o_n),
                           part(at::kFloat, {}, o_l)};
        at::Tensor work;
        if (size > 0) work = fresh({size}, at::kByte, *s);
        void *stream = stream_of(*s);
        if (unlocked(xtc_route_experts, T, E, (int64_t)top, static_cast<const void *>(s->data_ptr()), row_stride(*s),
                     static_cast<const uint8_t *>(data(mask)), as<int32_t>(r[0]), as<float>(r[1]), as<int32_t>(r[2]),
                     as<int32_t>(r[3]), as<int32_t>(r[4]), as<int32_t>(r[5]), as<float>(r[6]),
                     size > 0 ? work.data_ptr() : nullptr, size, dt, stream) != XTC_OK)
            Py_RETURN_NONE;
        return tuple_of(r);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// route_experts_backward(dp or None, scores, expert, p, counts, dloss, dtype or None): dscores
PyObject *route_experts_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[5];
    xtc_dtype dt;
    if (n != 7 || modes_active() || !tensors(args, t, 1) || !PyFloat_CheckExact(args[5])) Py_RETURN_NONE;
    const at::Tensor &s = *t[1], &e = *t[2], &p = *t[3], &counts = *t[4];
    if (!row_major(s) || !dtype_code(s, &dt) || e.dim() != 2) Py_RETURN_NONE;
    const int64_t T = s.size(0), E = s.size(1), top = e.size(1);
    if (!contiguous(e, at::kInt, {T, top}, s) || !contiguous(p, at::kFloat, {T, top}, s) ||
        !contiguous(counts, at::kInt, {E}, s) || (t[0] && !contiguous(*t[0], at::kFloat, {T, top}, s)))
        Py_RETURN_NONE;
    xtc_dtype code = dt;
    if (args[6] != Py_None) {
        if (!THPDtype_Check(args[6])) Py_RETURN_NONE;
        const at::ScalarType want = reinterpret_cast<THPDtype *>(args[6])->scalar_type;
        if (want != at::kFloat && want != at::kBFloat16) Py_RETURN_NONE;
        code = want == at::kFloat ? XTC_F32 : XTC_BF16;
    }
    try {
        const c10::DeviceGuard on(s.device());
        at::Tensor ds = fresh({T, E}, code == XTC_F32 ? at::kFloat : at::kBFloat16, s);
        void *stream = stream_of(s);
        if (unlocked(xtc_route_experts_backward, T, E, top, as<const float>(t[0]), static_cast<const void *>(s.data_ptr()),
                     row_stride(s), as<const int32_t>(e), as<const float>(p), as<const int32_t>(counts),
                     (float)PyFloat_AS_DOUBLE(args[5]), ds.data_ptr(), at_least_1(E), dt, code, stream) != XTC_OK)
            Py_RETURN_NONE;
        return wrapped(std::move(ds));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// combine_experts(rows, row, p or None, residual or None, dtype or None)
PyObject *combine_experts(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[4];
    if (n != 5 || modes_active() || !tensors(args, t, 4 | 8)) Py_RETURN_NONE;
    const at::Tensor &rows = *t[0], &row = *t[1];
    if (!row_major(rows) || !either(rows) || row.dim() != 2) Py_RETURN_NONE;
    const int64_t R = rows.size(0), D = rows.size(1), T = row.size(0), top = row.size(1);
    if (!contiguous(row, at::kInt, {T, top}, rows) || (t[2] && !contiguous(*t[2], at::kFloat, {T, top}, rows)) ||
        (t[3] && (!either(*t[3]) || !matrix(*t[3], t[3]->scalar_type(), T, D, rows))))
        Py_RETURN_NONE;
    try {
        const c10::DeviceGuard on(rows.device());
        at::Tensor out;
        xtc_dtype code;
        if (!result(nullptr, args[4], {T, D}, rows, &out, &code)) Py_RETURN_NONE;
        void *stream = stream_of(rows);
        if (unlocked(xtc_combine_experts, T, top, D, R, static_cast<const void *>(rows.data_ptr()),
                     R > 0 ? row_stride(rows) : at_least_1(D), as<const int32_t>(row), as<const float>(t[2]), data(t[3]),
                     t[3] ? row_stride(*t[3]) : 0, code_of(t[3]), out.data_ptr(), at_least_1(D), code_of(&rows), code,
                     stream) != XTC_OK)
            Py_RETURN_NONE;
        return wrapped(std::move(out));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// combine_experts_backward(dout, rows, row, token, p): (drows, dp)
PyObject *combine_experts_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    const at::Tensor *t[5];
    if (n != 5 || modes_active() || !tensors(args, t)) Py_RETURN_NONE;
    const at::Tensor &dout = *t[0], &rows = *t[1], &row = *t[2], &token = *t[3], &p = *t[4];
    if (!row_major(rows) || !either(rows) || !either(dout) || row.dim() != 2) Py_RETURN_NONE;
    const int64_t R = rows.size(0), D = rows.size(1), T = row.size(0), top = row.size(1);
    if (R != T * top || !contiguous(row, at::kInt, {T, top}, rows) || !contiguous(token, at::kInt, {R}, rows) ||
        !contiguous(p, at::kFloat, {T, top}, rows) || !matrix(dout, dout.scalar_type(), T, D, rows))
        Py_RETURN_NONE;
    try {
        const c10::DeviceGuard on(rows.device());
        at::Tensor drows = fresh({R, D}, rows.scalar_type(), rows), dp = fresh({T, top}, at::kFloat, rows);
        void *stream = stream_of(rows);
        if (unlocked(xtc_combine_experts_backward, T, top, D, static_cast<const void *>(dout.data_ptr()), row_stride(dout),
                     code_of(&dout), static_cast<const void *>(rows.data_ptr()), row_stride(rows), as<const int32_t>(row),
                     as<const int32_t>(token), as<const float>(p), drows.data_ptr(), at_least_1(D), as<float>(dp),
                     code_of(&rows), stream) != XTC_OK)
            Py_RETURN_NONE;
        return pair(std::move(drows), std::move(dp));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F));
}

PyMethodDef kMethods[] = {
    {"matmul", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&matmul)), METH_FASTCALL,
     "matmul(a, b, out, relu): the product, or None where the general path has to run"},
    {"conv2d_nchw", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&conv2d_nchw)), METH_FASTCALL,
     "conv2d_nchw(x, w, stride, pad, out, relu): the convolution, or None likewise"},
    {"rmsnorm", fast<rmsnorm>(), METH_FASTCALL, "rmsnorm(x, weight, residual, eps, quantize): its results, or None likewise"},
    {"rmsnorm_backward", fast<rmsnorm_backward>(), METH_FASTCALL, "rmsnorm_backward(dy, x, weight, rstd, dresidual)"},
    {"layernorm", fast<layernorm>(), METH_FASTCALL, "layernorm(x, weight, bias, residual, eps, quantize)"},
    {"layernorm_backward", fast<layernorm_backward>(), METH_FASTCALL, "layernorm_backward(dy, x, weight, mean, rstd, dresidual)"},
    {"quantize_fp8", fast<quantize_fp8>(), METH_FASTCALL, "quantize_fp8(x, block_rows)"},
    {"matmul_fp8", fast<matmul_fp8>(), METH_FASTCALL, "matmul_fp8(a, a_scale, b, b_scale, out, relu, dtype)"},
    {"linear", fast<linear>(), METH_FASTCALL, "linear(a, b, bias, residual, activation, transpose_b, keep, out, dtype)"},
    {"linear_wgrad", fast<linear_wgrad>(), METH_FASTCALL, "linear_wgrad(a, dy, out, dtype)"},
    {"activation_backward", fast<activation_backward>(), METH_FASTCALL, "activation_backward(dy, z, activation)"},
    {"matmul_grouped", fast<matmul_grouped>(), METH_FASTCALL, "matmul_grouped(a, b, ends, transpose_b, out, relu, dtype)"},
    {"matmul_grouped_wgrad", fast<matmul_grouped_wgrad>(), METH_FASTCALL, "matmul_grouped_wgrad(a, dy, ends, out, dtype)"},
    {"matmul_grouped_fp8", fast<matmul_grouped_fp8>(), METH_FASTCALL,
     "matmul_grouped_fp8(a, a_scale, b, b_scale, ends, out, relu, dtype)"},
    {"route_experts", fast<route_experts>(), METH_FASTCALL, "route_experts(scores, top, mask)"},
    {"route_experts_backward", fast<route_experts_backward>(), METH_FASTCALL,
     "route_experts_backward(dp, scores, expert, p, counts, dloss, dtype)"},
    {"combine_experts", fast<combine_experts>(), METH_FASTCALL, "combine_experts(rows, row, p, residual, dtype)"},
    {"combine_experts_backward", fast<combine_experts_backward>(), METH_FASTCALL,
     "combine_experts_backward(dout, rows, row, token, p)"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&kModule); }
