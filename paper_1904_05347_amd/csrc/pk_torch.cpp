// pk_torch.cpp -- the tensor calls of binding.py (gemm, conv2d_fwd,
// conv2d_winograd, the 8-bit and the attention operators) marshalled natively: torch tensors in, one
// C-ABI call on the current stream, the output tensor out.
//
// Every pointer is read before the interpreter lock is released: data_ptr()
// throws for a tensor without a storage, and an exception must not leave the
// part that runs without the lock.
//
// Why: a 64 x 64 x 64 product takes the GPU 4 us, the C-ABI call 0.8 us and
// its launch 2.9 us, but marshalled in Python (attribute reads, two ctypes
// calls, the allocations) a call took 12.5 us of host time, and that was the
// rate at which a program could issue small calls; marshalled here it takes
// 4.1 or 5.0 us (one or the other for the life of a process).
//
// Each function answers None whenever a call is anything but the plain case
// (a tensor subclass, an active torch mode, another type, device, layout or
// argument form, a shape that does not match, a C-ABI status that refuses the
// call): binding.py then runs its own checks and the same C-ABI call, so errors
// and unusual forms behave as they always did.  A failed launch is raised here:
// what went before it on the stream must not run twice.  Nothing is kept
// between calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/EmptyTensor.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <ATen/hip/impl/HIPCachingAllocatorMasqueradingAsCUDA.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstring>
#include <initializer_list>

#include "../../include/pk.h"

namespace {

// the C-ABI of the library binding.py loaded (set once by bind())
decltype(&pk_sgemm_ws) f_sgemm_ws;
decltype(&pk_sgemm_workspace_bytes_for) f_sgemm_workspace_bytes;
decltype(&pk_conv2d_fwd) f_conv2d_fwd;
decltype(&pk_conv2d_workspace_bytes_for) f_conv2d_workspace_bytes;
decltype(&pk_conv2d_out_dims) f_out_dims;
decltype(&pk_conv2d_same_pads) f_same_pads;
decltype(&pk_conv2d_winograd_tile_fwd) f_winograd;
decltype(&pk_conv2d_winograd_tile_workspace_bytes) f_winograd_workspace_bytes;
decltype(&pk_quantize_i8) f_quantize_i8;
decltype(&pk_rmsnorm_i8) f_rmsnorm_i8;
decltype(&pk_gated_i8) f_gated_i8;
decltype(&pk_dequantize_i8) f_dequantize_i8;
decltype(&pk_gemm_i8_ws) f_gemm_i8;
decltype(&pk_gemm_i8_workspace_bytes_for) f_gemm_i8_workspace_bytes;
decltype(&pk_rope_qk) f_rope_qk;
decltype(&pk_rope_qk_backward) f_rope_qk_backward;
decltype(&pk_rope_qk_backward_workspace_bytes) f_rope_qk_backward_workspace_bytes;
decltype(&pk_cache_append) f_cache_append;
decltype(&pk_attention_tree) f_attention_tree;
decltype(&pk_attention_tree_workspace_bytes) f_attention_tree_workspace_bytes;
PyObject *f_check;  // binding._check(status, entry point): raises

// The answer to a status other than PK_OK.
PyObject *refused(int st, const char *entry)
{
    if (st != PK_ERR_LAUNCH) Py_RETURN_NONE;
    return PyObject_CallFunction(f_check, "is", st, entry);
}

// A plain fp32 tensor on a GPU, or NULL.
const at::Tensor *plain(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.scalar_type() == at::kFloat && t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}

bool modes_active()
{
    return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set();
}

// Leading dimension of a row-major 2-D view whose rows do not overlap, or -1.
int64_t ld_2d(const at::Tensor &t)
{
    if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) return -1;
    if (t.size(0) > 1 && t.stride(0) < t.size(1)) return -1;
    return std::max<int64_t>(std::max(t.stride(0), t.size(1)), 1);
}

bool as_int(PyObject *o, int64_t *v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return !overflow;
}

bool as_float(PyObject *o, float *v)
{
    if (PyFloat_CheckExact(o)) {
        const double d = PyFloat_AS_DOUBLE(o);
        *v = (float)d;
        return *v != 0.f || d == 0.0;  // a beta that underflows isn't "no beta"
    }
    int64_t i;
    if (!as_int(o, &i) || i < -(1 << 24) || i > (1 << 24)) return false;
    *v = (float)i;
    return true;
}

// A workspace of at least `need` bytes, or the caller's: false when it is not
// a plain tensor.  `own` keeps an allocated one until the call has returned
// (the allocator reuses it in stream order).
bool workspace_for(PyObject *given, size_t need, const at::Tensor &like, at::Tensor *own, void **ptr, size_t *bytes)
{
    *ptr = nullptr;
    *bytes = 0;
    if (given != Py_None) {
        const at::Tensor *w = plain(given);
        if (!w) return false;
        *ptr = w->data_ptr();
        *bytes = (size_t)w->numel() * 4;
    } else if (need) {
        *own = at::empty({(int64_t)((need + 3) / 4)}, like.options().dtype(at::kFloat));
        *ptr = own->data_ptr();
        *bytes = (size_t)own->numel() * 4;
    }
    return true;
}

void *stream_of(const at::Tensor &t) { return (void *)c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

// gemm(a, b, c, alpha, beta, trans_a, trans_b, workspace)
PyObject *py_gemm(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    float alpha, beta;
    if (nargs != 8 || !PyBool_Check(args[5]) || !PyBool_Check(args[6]) || !as_float(args[3], &alpha) ||
        !as_float(args[4], &beta) || modes_active())
        Py_RETURN_NONE;
    const at::Tensor *a = plain(args[0]), *b = plain(args[1]);
    if (!a || !b) Py_RETURN_NONE;
    const bool ta = args[5] == Py_True, tb = args[6] == Py_True;
    const int64_t lda = ld_2d(*a), ldb = ld_2d(*b);
    if (lda < 0 || ldb < 0) Py_RETURN_NONE;
    const int64_t M = a->size(ta ? 1 : 0), K = a->size(ta ? 0 : 1), N = b->size(tb ? 0 : 1);
    if (b->size(tb ? 1 : 0) != K) Py_RETURN_NONE;
    at::Tensor c;
    const bool fresh = args[2] == Py_None;
    if (fresh) {
        if (beta != 0.f) Py_RETURN_NONE;
        c = at::empty({M, N}, a->options());
    } else {
        const at::Tensor *p = plain(args[2]);
        if (!p || p->dim() != 2 || p->size(0) != M || p->size(1) != N) Py_RETURN_NONE;
        c = *p;
    }
    const int64_t ldc = ld_2d(c);
    if (ldc < 0) Py_RETURN_NONE;
    const char fa = ta ? 'T' : 'N', fb = tb ? 'T' : 'N';
    const float *pa = (const float *)a->data_ptr(), *pb = (const float *)b->data_ptr();
    at::Tensor own;
    void *ws;
    size_t ws_bytes;
    const size_t need = args[7] == Py_None ? f_sgemm_workspace_bytes(fa, fb, M, N, K, pa, lda, pb, ldb, ldc) : 0;
    if (!workspace_for(args[7], need, *a, &own, &ws, &ws_bytes)) Py_RETURN_NONE;
    float *pc = (float *)c.data_ptr();
    void *stream = stream_of(c);
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_sgemm_ws(fa, fb, M, N, K, alpha, pa, lda, pb, ldb, beta, pc, ldc, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_sgemm_ws");
    if (fresh) return THPVariable_Wrap(std::move(c));
    Py_INCREF(args[2]);
    return args[2];
    END_HANDLE_TH_ERRORS
}

// The geometry both convolutions share, from x (N, H, W, Cin), w (KH, KW,
// Cin, Cout), a stride and a padding argument; false: not the plain case.
struct Geometry {
    const at::Tensor *x, *w;
    int64_t N, H, W, Cin, KH, KW, Cout, sh, sw, p[4], Ho, Wo;
};

bool geometry(PyObject *x, PyObject *w, PyObject *stride, PyObject *padding, Geometry *g)
{
    g->x = plain(x);
    g->w = plain(w);
    if (!g->x || !g->w || g->x->dim() != 4 || g->w->dim() != 4 || !g->x->is_contiguous() || !g->w->is_contiguous())
        return false;
    g->N = g->x->size(0);
    g->H = g->x->size(1);
    g->W = g->x->size(2);
    g->Cin = g->x->size(3);
    g->KH = g->w->size(0);
    g->KW = g->w->size(1);
    g->Cout = g->w->size(3);
    if (g->w->size(2) != g->Cin) return false;
    if (stride == Py_None) {
        g->sh = g->sw = 1;
    } else if (PyLong_CheckExact(stride)) {
        if (!as_int(stride, &g->sh)) return false;
        g->sw = g->sh;
    } else if (!PyTuple_CheckExact(stride) || PyTuple_GET_SIZE(stride) != 2 ||
               !as_int(PyTuple_GET_ITEM(stride, 0), &g->sh) || !as_int(PyTuple_GET_ITEM(stride, 1), &g->sw)) {
        return false;
    }
    if (PyUnicode_CheckExact(padding)) {
        if (PyUnicode_CompareWithASCIIString(padding, "SAME") == 0) {
            if (f_same_pads(g->H, g->W, g->KH, g->KW, g->sh, g->sw, g->p) != PK_OK) return false;
        } else if (PyUnicode_CompareWithASCIIString(padding, "VALID") == 0) {
            memset(g->p, 0, sizeof(g->p));
        } else {
            return false;
        }
    } else {
        if (!PyTuple_CheckExact(padding) || PyTuple_GET_SIZE(padding) != 4) return false;
        for (int i = 0; i < 4; ++i)
            if (!as_int(PyTuple_GET_ITEM(padding, i), &g->p[i])) return false;
    }
    return f_out_dims(g->H, g->W, g->KH, g->KW, g->sh, g->sw, g->p[0], g->p[1], g->p[2], g->p[3], &g->Ho, &g->Wo) ==
           PK_OK;
}

// The output tensor: the caller's (plain, contiguous, of this shape) or a new one.
bool output_for(PyObject *given, const Geometry &g, at::Tensor *y)
{
    if (given == Py_None) {
        *y = at::empty({g.N, g.Ho, g.Wo, g.Cout}, g.x->options());
        return true;
    }
    const at::Tensor *p = plain(given);
    if (!p || p->dim() != 4 || p->size(0) != g.N || p->size(1) != g.Ho || p->size(2) != g.Wo || p->size(3) != g.Cout ||
        !p->is_contiguous())
        return false;
    *y = *p;
    return true;
}

PyObject *answer(PyObject *given, at::Tensor &&y)
{
    if (given == Py_None) return THPVariable_Wrap(std::move(y));
    Py_INCREF(given);
    return given;
}

// conv2d_fwd(x, w, stride, padding, out, workspace)
PyObject *py_conv2d_fwd(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    Geometry g;
    at::Tensor y, own;
    if (nargs != 6 || args[2] == Py_None || modes_active() || !geometry(args[0], args[1], args[2], args[3], &g) ||
        !output_for(args[4], g, &y))
        Py_RETURN_NONE;
    const float *px = (const float *)g.x->data_ptr(), *pw = (const float *)g.w->data_ptr();
    const size_t need = args[5] == Py_None
                            ? f_conv2d_workspace_bytes(px, g.N, g.H, g.W, g.Cin, pw, g.KH, g.KW, g.Cout, g.sh, g.sw,
                                                       g.p[0], g.p[1], g.p[2], g.p[3])
                            : 0;
    void *ws;
    size_t ws_bytes;
    if (!workspace_for(args[5], need, *g.x, &own, &ws, &ws_bytes)) Py_RETURN_NONE;
    float *py = (float *)y.data_ptr();
    void *stream = stream_of(y);
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_conv2d_fwd(px, g.N, g.H, g.W, g.Cin, pw, g.KH, g.KW, g.Cout, g.sh, g.sw, g.p[0], g.p[1], g.p[2], g.p[3],
                      py, g.Ho, g.Wo, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_conv2d_fwd");
    return answer(args[4], std::move(y));
    END_HANDLE_TH_ERRORS
}

// conv2d_winograd(x, w, padding, out, workspace, tile)
PyObject *py_conv2d_winograd(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    Geometry g;
    at::Tensor y, own;
    int64_t m;
    if (nargs != 6 || !as_int(args[5], &m) || modes_active() ||
        !geometry(args[0], args[1], Py_None, args[2], &g) || !output_for(args[3], g, &y))
        Py_RETURN_NONE;
    size_t need = 0;
    if (args[4] == Py_None) {
        need = f_winograd_workspace_bytes(m, g.N, g.H, g.W, g.Cin, g.Cout, g.p[0], g.p[1], g.p[2], g.p[3]);
        if (need < 4) need = 4;
    }
    void *ws;
    size_t ws_bytes;
    if (!workspace_for(args[4], need, *g.x, &own, &ws, &ws_bytes)) Py_RETURN_NONE;
    const float *px = (const float *)g.x->data_ptr(), *pw = (const float *)g.w->data_ptr();
    float *py = (float *)y.data_ptr();
    void *stream = stream_of(y);
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_winograd(px, g.N, g.H, g.W, g.Cin, pw, g.KH, g.KW, g.Cout, 1, 1, g.p[0], g.p[1], g.p[2], g.p[3], py, g.Ho,
                    g.Wo, m, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_conv2d_winograd_tile_fwd");
    return answer(args[3], std::move(y));
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------- 8-bit operators

int dtype_code(at::ScalarType t)
{
    return t == at::kFloat ? PK_F32 : t == at::kBFloat16 ? PK_BF16 : t == at::kHalf ? PK_F16 : -1;
}

// A plain strided tensor on a GPU, or NULL.  A transform's wrapper (torch.func)
// has the type and answers of a plain tensor, but no storage; a negative view
// (the imaginary part of a conjugate) has its values' negatives there.
const at::Tensor *on_gpu(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && !t.is_neg() ? &t : nullptr;
}

// A plain matrix of float32, bfloat16 or float16, with its code and leading dimension.
const at::Tensor *matrix(PyObject *o, int *code, int64_t *ld)
{
    const at::Tensor *t = on_gpu(o);
    if (!t || (*code = dtype_code(t->scalar_type())) < 0 || (*ld = ld_2d(*t)) < 0) return nullptr;
    return t;
}

const at::Tensor *matrix_i8(PyObject *o, int64_t *ld)
{
    const at::Tensor *t = on_gpu(o);
    return t && t->scalar_type() == at::kChar && (*ld = ld_2d(*t)) >= 0 ? t : nullptr;
}

// A contiguous vector of n elements of this type on that device.
const at::Tensor *vec(PyObject *o, int64_t n, at::ScalarType type, const at::Tensor &like)
{
    const at::Tensor *t = on_gpu(o);
    if (!t || t->scalar_type() != type || t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1) ||
        t->device() != like.device())
        return nullptr;
    return t;
}

// A new tensor on that device.  Made without torch's dispatcher where the device
// is the current one (0.5 us a tensor instead of 1.0, and a call makes up to three):
// no mode is active here that could have a say, and every operand has a storage.
at::Tensor fresh(at::IntArrayRef size, at::IntArrayRef stride, at::ScalarType type, const at::Tensor &like)
{
    if (like.device().index() != c10::hip::current_device())
        return at::empty_strided(size, stride, like.options().dtype(type));
    return at::Tensor(at::detail::empty_strided_generic(size, stride,
                                                        c10::hip::HIPCachingAllocatorMasqueradingAsCUDA::get(),
                                                        c10::DispatchKeySet(c10::DispatchKey::CUDA), type));
}

at::Tensor fresh_matrix(int64_t M, int64_t N, at::ScalarType type, const at::Tensor &like)
{
    return fresh({M, N}, {std::max<int64_t>(N, 1), 1}, type, like);
}

bool same_shape(const at::Tensor &t, int64_t M, int64_t N, const at::Tensor &like)
{
    return t.dim() == 2 && t.size(0) == M && t.size(1) == N && t.device() == like.device();
}

// The 8-bit output and its scales: the caller's, or new ones whose rows start
// at multiples of 16 bytes, long ones at memory lines of 128.
struct RowsOut {
    at::Tensor q, scale;
    int64_t ld;
};

bool rows_out(PyObject *out, PyObject *scale, int64_t M, int64_t N, const at::Tensor &like, RowsOut *r)
{
    if (out == Py_None) {
        const int64_t step = N >= 1024 ? 128 : 16;
        r->ld = std::max<int64_t>(1, (N + step - 1) / step * step);
        r->q = fresh({M, N}, {r->ld, 1}, at::kChar, like);
    } else {
        const at::Tensor *t = matrix_i8(out, &r->ld);
        if (!t || !same_shape(*t, M, N, like)) return false;
        r->q = *t;
    }
    if (scale == Py_None) {
        r->scale = fresh({M}, {1}, at::kFloat, like);
    } else {
        const at::Tensor *t = vec(scale, M, at::kFloat, like);
        if (!t) return false;
        r->scale = *t;
    }
    return true;
}

// `given`, or the new tensor in its place.
PyObject *given_or(PyObject *given, at::Tensor &&t)
{
    if (given == Py_None) return THPVariable_Wrap(std::move(t));
    Py_INCREF(given);
    return given;
}

PyObject *pair(PyObject *out, PyObject *scale, RowsOut &&r)
{
    PyObject *a = given_or(out, std::move(r.q)), *b = a ? given_or(scale, std::move(r.scale)) : nullptr;
    PyObject *t = b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return t;
}

// quantize_i8(x, out, scale)
PyObject *py_quantize_i8(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int dt;
    int64_t ldx;
    RowsOut r;
    if (nargs != 3 || modes_active()) Py_RETURN_NONE;
    const at::Tensor *x = matrix(args[0], &dt, &ldx);
    if (!x || !rows_out(args[1], args[2], x->size(0), x->size(1), *x, &r)) Py_RETURN_NONE;
    void *stream = stream_of(*x), *px = x->data_ptr();
    const int64_t M = x->size(0), N = x->size(1);
    int8_t *q = (int8_t *)r.q.data_ptr();
    float *scale = (float *)r.scale.data_ptr();
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_quantize_i8(px, dt, M, N, ldx, q, r.ld, scale, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_quantize_i8");
    return pair(args[1], args[2], std::move(r));
    END_HANDLE_TH_ERRORS
}

// rmsnorm_i8(x, weight, residual, eps, sum_out, out, scale)
PyObject *py_rmsnorm_i8(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int dt, dr, wt;
    int64_t ldx, ldr = 0, lds = 0;
    float eps;
    RowsOut r;
    if (nargs != 7 || !as_float(args[3], &eps) || modes_active()) Py_RETURN_NONE;
    const at::Tensor *x = matrix(args[0], &dt, &ldx), *w = on_gpu(args[1]), *res = nullptr;
    if (!x || !w) Py_RETURN_NONE;
    const int64_t M = x->size(0), N = x->size(1);
    wt = dtype_code(w->scalar_type());
    if ((wt != dt && wt != PK_F32) || !vec(args[1], N, w->scalar_type(), *x)) Py_RETURN_NONE;
    at::Tensor sum;
    if (args[2] == Py_None) {
        if (args[4] != Py_None) Py_RETURN_NONE;
    } else {
        res = matrix(args[2], &dr, &ldr);
        if (!res || dr != dt || !same_shape(*res, M, N, *x)) Py_RETURN_NONE;
        if (args[4] == Py_None) {
            sum = fresh_matrix(M, N, x->scalar_type(), *x);
            lds = std::max<int64_t>(N, 1);
        } else {
            const at::Tensor *t = matrix(args[4], &dr, &lds);
            if (!t || dr != dt || !same_shape(*t, M, N, *x)) Py_RETURN_NONE;
            sum = *t;
        }
    }
    if (!rows_out(args[5], args[6], M, N, *x, &r)) Py_RETURN_NONE;
    void *stream = stream_of(*x), *px = x->data_ptr(), *pr = res ? res->data_ptr() : nullptr, *pw = w->data_ptr(),
         *ps = res ? sum.data_ptr() : nullptr;
    int8_t *q = (int8_t *)r.q.data_ptr();
    float *scale = (float *)r.scale.data_ptr();
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_rmsnorm_i8(px, dt, M, N, ldx, pr, ldr, pw, wt, eps, ps, lds, q, r.ld, scale, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_rmsnorm_i8");
    PyObject *a = given_or(args[5], std::move(r.q)), *b = a ? given_or(args[6], std::move(r.scale)) : nullptr;
    PyObject *c = !b ? nullptr : res ? given_or(args[4], std::move(sum)) : given_or(args[0], at::Tensor());
    PyObject *t = c ? PyTuple_Pack(3, a, b, c) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    Py_XDECREF(c);
    return t;
    END_HANDLE_TH_ERRORS
}

// gated_i8(gate, up, activation, out, scale)
PyObject *py_gated_i8(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int dt, du;
    int64_t ldg, ldu;
    RowsOut r;
    if (nargs != 5 || !PyUnicode_CheckExact(args[2]) || modes_active()) Py_RETURN_NONE;
    const int act = PyUnicode_CompareWithASCIIString(args[2], "silu") == 0   ? PK_ACT_SILU
                    : PyUnicode_CompareWithASCIIString(args[2], "gelu") == 0 ? PK_ACT_GELU
                                                                             : -1;
    const at::Tensor *gate = matrix(args[0], &dt, &ldg), *up = matrix(args[1], &du, &ldu);
    if (act < 0 || !gate || !up || du != dt || !same_shape(*up, gate->size(0), gate->size(1), *gate)) Py_RETURN_NONE;
    if (!rows_out(args[3], args[4], gate->size(0), gate->size(1), *gate, &r)) Py_RETURN_NONE;
    void *stream = stream_of(*gate), *pg = gate->data_ptr(), *pu = up->data_ptr();
    const int64_t M = gate->size(0), N = gate->size(1);
    int8_t *q = (int8_t *)r.q.data_ptr();
    float *scale = (float *)r.scale.data_ptr();
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_gated_i8(pg, ldg, pu, ldu, dt, act, M, N, q, r.ld, scale, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_gated_i8");
    return pair(args[3], args[4], std::move(r));
    END_HANDLE_TH_ERRORS
}

// The floating output of M x N: the caller's, or a new one of the type asked
// for (`standard` when none is).
bool float_out(PyObject *out, PyObject *dtype, at::ScalarType standard, int64_t M, int64_t N, const at::Tensor &like,
               at::Tensor *t, int *code, int64_t *ld)
{
    if (dtype != Py_None && !THPDtype_Check(dtype)) return false;
    if (out == Py_None) {
        const at::ScalarType type = dtype == Py_None ? standard : ((THPDtype *)dtype)->scalar_type;
        if ((*code = dtype_code(type)) < 0) return false;
        *t = fresh_matrix(M, N, type, like);
        *ld = std::max<int64_t>(N, 1);
        return true;
    }
    const at::Tensor *p = matrix(out, code, ld);
    if (!p || (dtype != Py_None && p->scalar_type() != ((THPDtype *)dtype)->scalar_type) || !same_shape(*p, M, N, like))
        return false;
    *t = *p;
    return true;
}

// dequantize_i8(q, scale, dtype, out)
PyObject *py_dequantize_i8(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int dt;
    int64_t ldq, ldx;
    at::Tensor x;
    if (nargs != 4 || modes_active()) Py_RETURN_NONE;
    const at::Tensor *q = matrix_i8(args[0], &ldq);
    if (!q) Py_RETURN_NONE;
    const int64_t M = q->size(0), N = q->size(1);
    const at::Tensor *scale = vec(args[1], M, at::kFloat, *q);
    if (!scale || !float_out(args[3], args[2], at::kFloat, M, N, *q, &x, &dt, &ldx)) Py_RETURN_NONE;
    void *stream = stream_of(*q), *px = x.data_ptr();
    const int8_t *pq = (const int8_t *)q->data_ptr();
    const float *ps = (const float *)scale->data_ptr();
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_dequantize_i8(pq, ldq, ps, M, N, px, dt, ldx, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_dequantize_i8");
    return given_or(args[3], std::move(x));
    END_HANDLE_TH_ERRORS
}

// gemm_i8(a, b, a_scale, b_scale, bias, dtype, out, workspace)
PyObject *py_gemm_i8(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int dt;
    int64_t lda, ldb, ldc;
    at::Tensor c, own;
    if (nargs != 8 || modes_active()) Py_RETURN_NONE;
    const at::Tensor *a = matrix_i8(args[0], &lda), *b = matrix_i8(args[1], &ldb), *bias = nullptr;
    if (!a || !b || a->size(1) != b->size(1) || a->device() != b->device()) Py_RETURN_NONE;
    const int64_t M = a->size(0), N = b->size(0), K = a->size(1);
    const at::Tensor *sa = vec(args[2], M, at::kFloat, *a), *sb = vec(args[3], N, at::kFloat, *a);
    if (!sa || !sb || (args[4] != Py_None && !(bias = vec(args[4], N, at::kFloat, *a)))) Py_RETURN_NONE;
    if (!float_out(args[6], args[5], at::kBFloat16, M, N, *a, &c, &dt, &ldc)) Py_RETURN_NONE;
    const int8_t *pa = (const int8_t *)a->data_ptr(), *pb = (const int8_t *)b->data_ptr();
    const size_t need = args[7] == Py_None ? f_gemm_i8_workspace_bytes(M, N, K, pa, lda, pb, ldb) : 0;
    void *ws;
    size_t ws_bytes;
    if (args[7] != Py_None) {
        const at::Tensor *w = plain(args[7]);
        if (!w || !w->is_contiguous() || w->device() != a->device()) Py_RETURN_NONE;
    }
    if (!workspace_for(args[7], need, *a, &own, &ws, &ws_bytes)) Py_RETURN_NONE;
    void *stream = stream_of(*a), *pc = c.data_ptr();
    const float *psa = (const float *)sa->data_ptr(), *psb = (const float *)sb->data_ptr(),
                *pbias = bias ? (const float *)bias->data_ptr() : nullptr;
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_gemm_i8(M, N, K, pa, lda, psa, pb, ldb, psb, pbias, pc, dt, ldc, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_gemm_i8_ws");
    return given_or(args[6], std::move(c));
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------- attention operators

// A plain tensor of tokens x heads x channels, its channels contiguous.
const at::Tensor *heads(PyObject *o, pk_heads *h)
{
    const at::Tensor *t = on_gpu(o);
    if (!t || t->dim() != 3 || (t->size(2) > 1 && t->stride(2) != 1)) return nullptr;
    *h = {t->data_ptr(), t->size(1), t->stride(0), t->stride(1)};
    return t;
}

// The same, of `like`'s type, device, tokens and channels.
const at::Tensor *heads_like(PyObject *o, const at::Tensor &like, pk_heads *h)
{
    const at::Tensor *t = heads(o, h);
    return t && t->scalar_type() == like.scalar_type() && t->device() == like.device() && t->size(0) == like.size(0) &&
                   t->size(2) == like.size(2)
               ? t : nullptr;
}

// An output of `like`'s shape: the caller's, or a new one.
bool heads_out(PyObject *o, const at::Tensor &like, at::Tensor *t, pk_heads *h)
{
    if (o != Py_None) {
        const at::Tensor *given = heads_like(o, like, h);
        if (!given || given->size(1) != like.size(1)) return false;
        *t = *given;
        return true;
    }
    const int64_t H = like.size(1), d = like.size(2), row = std::max<int64_t>(H * d, 1), step = std::max<int64_t>(d, 1);
    *t = fresh({like.size(0), H, d}, {row, step, 1}, like.scalar_type(), like);
    *h = {t->data_ptr(), H, row, step};
    return true;
}

bool pages_of(PyObject *key, PyObject *value, const at::Tensor &like, pk_cache *c)
{
    const at::Tensor *k = on_gpu(key), *v = on_gpu(value);
    if (!k || !v || k->dim() != 4 || v->dim() != 4 || k->sizes() != v->sizes() || k->size(3) != like.size(2)) return false;
    if (k->scalar_type() != like.scalar_type() || v->scalar_type() != like.scalar_type() || k->device() != like.device() ||
        v->device() != like.device() || (k->size(3) > 1 && (k->stride(3) != 1 || v->stride(3) != 1)))
        return false;
    *c = {k->data_ptr(), v->data_ptr(), k->size(0), k->size(1), k->size(2),
          {k->stride(0), k->stride(1), k->stride(2)}, {v->stride(0), v->stride(1), v->stride(2)}};
    return true;
}

// Both None (*rot is NULL then), or positions and frequencies of these tokens.
bool rotation(PyObject *positions, PyObject *frequencies, PyObject *layout, PyObject *amplitude, const at::Tensor &like,
              pk_rotation *r, const pk_rotation **rot)
{
    *rot = nullptr;
    if (!PyUnicode_CheckExact(layout)) return false;
    r->interleaved = PyUnicode_CompareWithASCIIString(layout, "interleaved") == 0;
    if (!r->interleaved && PyUnicode_CompareWithASCIIString(layout, "half") != 0) return false;
    if (!as_float(amplitude, &r->amplitude)) return false;
    if (positions == Py_None && frequencies == Py_None) return true;
    const at::Tensor *f = on_gpu(frequencies), *p = vec(positions, like.size(0), at::kLong, like);
    if (!f || !p || f->dim() != 1 || !vec(frequencies, f->size(0), at::kDouble, like) || 2 * f->size(0) > like.size(2)) return false;
    r->positions = (const int64_t *)p->data_ptr();
    r->frequencies = (const double *)f->data_ptr();
    r->pairs = f->size(0);
    *rot = r;
    return true;
}

// The norms' weights, of one type: the heads' or fp32.
struct Weights {
    const at::Tensor *t[2];
    const void *p[2];
    int code;
};

bool weights(PyObject *q, PyObject *k, const at::Tensor &like, Weights *w)
{
    *w = {{nullptr, nullptr}, {nullptr, nullptr}, PK_F32};
    PyObject *given[2] = {q, k};
    for (int i = 0; i < 2; ++i) {
        if (given[i] == Py_None) continue;
        const at::Tensor *t = on_gpu(given[i]);
        if (!t || (t->scalar_type() != like.scalar_type() && t->scalar_type() != at::kFloat)) return false;
        if (!vec(given[i], like.size(2), t->scalar_type(), like)) return false;
        const int code = dtype_code(t->scalar_type());
        if ((w->t[0] || w->t[1]) && code != w->code) return false;
        w->code = code;
        w->t[i] = t;
        w->p[i] = t->data_ptr();
    }
    return true;
}

// `given`, or the new tensor in its place; None where there is neither.
PyObject *given_or_none(PyObject *given, at::Tensor &&t)
{
    if (given == Py_None && !t.defined()) Py_RETURN_NONE;
    return given_or(given, std::move(t));
}

PyObject *tuple_of(std::initializer_list<PyObject *> parts)
{
    PyObject *t = PyTuple_New((Py_ssize_t)parts.size());
    Py_ssize_t i = 0;
    bool whole = t != nullptr;
    for (PyObject *p : parts) {
        if (!p) whole = false;
        if (t)
            PyTuple_SET_ITEM(t, i++, p);  // NULL is no value of a finished tuple: it is dropped below
        else
            Py_XDECREF(p);
    }
    if (!whole) Py_CLEAR(t);
    return t;
}

// rope_qk(q, k, positions, frequencies, q_weight, k_weight, eps, layout, amplitude, q_out, k_out)
PyObject *py_rope_qk(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    pk_heads hq, hk, oq, ok;
    pk_rotation r;
    const pk_rotation *rot;
    Weights w;
    float eps;
    at::Tensor out_q, out_k;
    if (nargs != 11 || !as_float(args[6], &eps) || modes_active()) Py_RETURN_NONE;
    const at::Tensor *q = heads(args[0], &hq), *k = nullptr;
    if (!q) Py_RETURN_NONE;
    const int dt = dtype_code(q->scalar_type());
    if (dt < 0 || !rotation(args[2], args[3], args[7], args[8], *q, &r, &rot) || !weights(args[4], args[5], *q, &w)) Py_RETURN_NONE;
    if (args[1] != Py_None) {
        k = heads_like(args[1], *q, &hk);
        if (!k || !heads_out(args[10], *k, &out_k, &ok)) Py_RETURN_NONE;
    } else if (args[5] != Py_None || args[10] != Py_None) {
        Py_RETURN_NONE;
    }
    if (!heads_out(args[9], *q, &out_q, &oq)) Py_RETURN_NONE;
    const int64_t M = q->size(0), d = q->size(2);
    const pk_heads *ph = k ? &hk : nullptr, *po = k ? &ok : nullptr;
    const void *qw = w.p[0], *kw = w.p[1];
    const int wt = w.code;
    void *stream = stream_of(*q);
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_rope_qk(dt, M, d, &hq, ph, rot, qw, kw, wt, eps, &oq, po, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_rope_qk");
    return tuple_of({given_or(args[9], std::move(out_q)), given_or_none(args[10], std::move(out_k))});
    END_HANDLE_TH_ERRORS
}

// rope_qk_backward(dq, dk, q, k, positions, frequencies, q_weight, k_weight, eps, layout, amplitude, q_grad, k_grad)
PyObject *py_rope_qk_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    pk_heads hdq, hdk, hq, hk, gq, gk;
    pk_rotation r;
    const pk_rotation *rot;
    Weights w;
    float eps;
    at::Tensor out_q, out_k, wgrad[2], own;
    if (nargs != 13 || !as_float(args[8], &eps) || modes_active()) Py_RETURN_NONE;
    const at::Tensor *dq = heads(args[0], &hdq), *dk = nullptr;
    if (!dq) Py_RETURN_NONE;
    const int dt = dtype_code(dq->scalar_type());
    if (dt < 0 || !rotation(args[4], args[5], args[9], args[10], *dq, &r, &rot) || !weights(args[6], args[7], *dq, &w)) Py_RETURN_NONE;
    if (args[1] != Py_None) {
        dk = heads_like(args[1], *dq, &hdk);
        if (!dk || !heads_out(args[12], *dk, &out_k, &gk)) Py_RETURN_NONE;
    } else if (args[7] != Py_None || args[12] != Py_None) {
        Py_RETURN_NONE;
    }
    if (!heads_out(args[11], *dq, &out_q, &gq)) Py_RETURN_NONE;
    // the inputs, where a weight needs them
    const pk_heads *pq = nullptr, *pk = nullptr;
    if (w.t[0]) {
        const at::Tensor *q = heads_like(args[2], *dq, &hq);
        if (!q || q->size(1) != dq->size(1)) Py_RETURN_NONE;
        pq = &hq;
    }
    if (w.t[1]) {
        const at::Tensor *k = heads_like(args[3], *dk, &hk);
        if (!k || k->size(1) != dk->size(1)) Py_RETURN_NONE;
        pk = &hk;
    }
    const int64_t M = dq->size(0), d = dq->size(2);
    void *wg[2] = {nullptr, nullptr}, *ws = nullptr;
    for (int i = 0; i < 2; ++i) {
        if (!w.t[i]) continue;
        wgrad[i] = fresh({d}, {1}, w.t[i]->scalar_type(), *dq);
        wg[i] = wgrad[i].data_ptr();
    }
    size_t bytes = w.t[0] || w.t[1] ? f_rope_qk_backward_workspace_bytes(M, d) : 0;
    if (bytes) {
        own = fresh({(int64_t)(bytes / 4)}, {1}, at::kFloat, *dq);
        ws = own.data_ptr();
    }
    const pk_heads *pdk = dk ? &hdk : nullptr, *pgk = dk ? &gk : nullptr;
    const void *qw = w.p[0], *kw = w.p[1];
    const int wt = w.code;
    void *gqw = wg[0], *gkw = wg[1], *stream = stream_of(*dq);
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_rope_qk_backward(dt, M, d, &hdq, pdk, pq, pk, rot, qw, kw, wt, eps, &gq, pgk, gqw, gkw, ws, bytes, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_rope_qk_backward");
    return tuple_of({given_or(args[11], std::move(out_q)), given_or_none(args[12], std::move(out_k)),
                     given_or_none(Py_None, std::move(wgrad[0])), given_or_none(Py_None, std::move(wgrad[1]))});
    END_HANDLE_TH_ERRORS
}

// cache_append(k, v, key_cache, value_cache, slots, positions, frequencies, k_weight, q, q_weight, eps, layout, amplitude, q_out):
// (q_out,), which tells a call without queries from one that was not made
PyObject *py_cache_append(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    pk_heads hq, hk, hv, oq;
    pk_cache cache;
    pk_rotation r;
    const pk_rotation *rot;
    Weights w;
    float eps;
    at::Tensor out_q;
    if (nargs != 14 || !as_float(args[10], &eps) || modes_active()) Py_RETURN_NONE;
    const at::Tensor *k = heads(args[0], &hk), *q = nullptr;
    if (!k) Py_RETURN_NONE;
    const int dt = dtype_code(k->scalar_type());
    const at::Tensor *v = heads_like(args[1], *k, &hv);
    if (dt < 0 || !v || v->size(1) != k->size(1) || !pages_of(args[2], args[3], *k, &cache) || cache.heads != k->size(1)) Py_RETURN_NONE;
    const at::Tensor *slots = vec(args[4], k->size(0), at::kLong, *k);
    if (!slots || !rotation(args[5], args[6], args[11], args[12], *k, &r, &rot) || !weights(args[9], args[7], *k, &w)) Py_RETURN_NONE;
    if (args[8] != Py_None) {
        q = heads_like(args[8], *k, &hq);
        if (!q || !heads_out(args[13], *q, &out_q, &oq)) Py_RETURN_NONE;
    } else if (args[9] != Py_None || args[13] != Py_None) {
        Py_RETURN_NONE;
    }
    const int64_t M = k->size(0), d = k->size(2), *at = (const int64_t *)slots->data_ptr();
    const pk_heads *ph = q ? &hq : nullptr, *po = q ? &oq : nullptr;
    const void *qw = w.p[0], *kw = w.p[1];
    const int wt = w.code;
    void *stream = stream_of(*k);
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_cache_append(dt, M, d, ph, &hk, &hv, rot, qw, kw, wt, eps, po, &cache, at, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_cache_append");
    return tuple_of({given_or_none(args[13], std::move(out_q))});
    END_HANDLE_TH_ERRORS
}

// attention_tree(q, key_cache, value_cache, page_table, lengths, starts, most, mask, scale, cap, out, lse, workspace)
PyObject *py_attention_tree(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    pk_heads hq, ho;
    pk_cache cache;
    int64_t most, ld_table, ld_lse = 0;
    float scale, cap;
    at::Tensor out, sums, own;
    if (nargs != 13 || !as_int(args[6], &most) || !as_float(args[9], &cap) || modes_active()) Py_RETURN_NONE;
    const at::Tensor *q = heads(args[0], &hq);
    if (!q) Py_RETURN_NONE;
    const int dt = dtype_code(q->scalar_type());
    if (dt < 0 || !pages_of(args[1], args[2], *q, &cache)) Py_RETURN_NONE;
    const int64_t M = q->size(0), Hq = q->size(1), d = q->size(2);
    if (args[8] == Py_None)
        scale = (float)std::pow((double)std::max<int64_t>(d, 1), -0.5);
    else if (!as_float(args[8], &scale))
        Py_RETURN_NONE;
    const at::Tensor *table = on_gpu(args[3]);
    if (!table || table->scalar_type() != at::kInt || table->device() != q->device() || (ld_table = ld_2d(*table)) < 0) Py_RETURN_NONE;
    const int64_t B = table->size(0), P = table->size(1);
    const at::Tensor *lengths = vec(args[4], B, at::kInt, *q), *starts = vec(args[5], B + 1, at::kInt, *q), *mask = nullptr;
    if (!lengths || !starts || (args[7] != Py_None && !(mask = vec(args[7], M, at::kLong, *q)))) Py_RETURN_NONE;
    if (!heads_out(args[10], *q, &out, &ho)) Py_RETURN_NONE;
    const bool none = args[11] == Py_None || args[11] == Py_False, made = args[11] == Py_True;
    if (made) {
        sums = fresh_matrix(M, Hq, at::kFloat, *q);
        ld_lse = std::max<int64_t>(Hq, 1);
    } else if (!none) {
        const at::Tensor *t = on_gpu(args[11]);
        if (!t || t->scalar_type() != at::kFloat || (ld_lse = ld_2d(*t)) < 0 || !same_shape(*t, M, Hq, *q)) Py_RETURN_NONE;
        sums = *t;
    }
    void *ws = nullptr;
    size_t bytes = 0;
    if (args[12] != Py_None) {
        const at::Tensor *t = plain(args[12]);
        if (!t || !t->is_contiguous() || t->device() != q->device()) Py_RETURN_NONE;
        ws = t->data_ptr();
        bytes = (size_t)t->numel() * 4;
    } else if ((bytes = f_attention_tree_workspace_bytes(dt, d, Hq, cache.heads, B, P, cache.page_size, most)) != 0) {
        own = fresh({(int64_t)(bytes / 4)}, {1}, at::kFloat, *q);
        ws = own.data_ptr();
    }
    const int32_t *pt = (const int32_t *)table->data_ptr(), *pl = (const int32_t *)lengths->data_ptr(),
                  *ps = (const int32_t *)starts->data_ptr();
    const uint64_t *pm = mask ? (const uint64_t *)mask->data_ptr() : nullptr;
    float *lse = none ? nullptr : (float *)sums.data_ptr();
    void *stream = stream_of(*q);
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f_attention_tree(dt, M, d, &hq, &cache, pt, B, P, ld_table, pl, ps, most, pm, scale, cap, &ho, lse, ld_lse, ws, bytes, stream);
    Py_END_ALLOW_THREADS
    if (st != PK_OK) return refused(st, "pk_attention_tree");
    PyObject *o = given_or(args[10], std::move(out));
    if (none || !o) return o;
    return tuple_of({o, given_or(made ? Py_None : args[11], std::move(sums))});
    END_HANDLE_TH_ERRORS
}

// bind(addresses, check): the entry points above, in their order, and the
// function that raises for a status.
PyObject *py_bind(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    constexpr int kEntries = 20;
    if (nargs != kEntries + 1) {
        PyErr_SetString(PyExc_TypeError, "bind takes the addresses of twenty entry points and a function");
        return nullptr;
    }
    void *p[kEntries];
    for (int i = 0; i < kEntries; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
            return nullptr;
        }
    }
    f_sgemm_ws = (decltype(f_sgemm_ws))p[0];
    f_sgemm_workspace_bytes = (decltype(f_sgemm_workspace_bytes))p[1];
    f_conv2d_fwd = (decltype(f_conv2d_fwd))p[2];
    f_conv2d_workspace_bytes = (decltype(f_conv2d_workspace_bytes))p[3];
    f_out_dims = (decltype(f_out_dims))p[4];
    f_same_pads = (decltype(f_same_pads))p[5];
    f_winograd = (decltype(f_winograd))p[6];
    f_winograd_workspace_bytes = (decltype(f_winograd_workspace_bytes))p[7];
    f_quantize_i8 = (decltype(f_quantize_i8))p[8];
    f_rmsnorm_i8 = (decltype(f_rmsnorm_i8))p[9];
    f_gated_i8 = (decltype(f_gated_i8))p[10];
    f_dequantize_i8 = (decltype(f_dequantize_i8))p[11];
    f_gemm_i8 = (decltype(f_gemm_i8))p[12];
    f_gemm_i8_workspace_bytes = (decltype(f_gemm_i8_workspace_bytes))p[13];
    f_rope_qk = (decltype(f_rope_qk))p[14];
    f_rope_qk_backward = (decltype(f_rope_qk_backward))p[15];
    f_rope_qk_backward_workspace_bytes = (decltype(f_rope_qk_backward_workspace_bytes))p[16];
    f_cache_append = (decltype(f_cache_append))p[17];
    f_attention_tree = (decltype(f_attention_tree))p[18];
    f_attention_tree_workspace_bytes = (decltype(f_attention_tree_workspace_bytes))p[19];
    Py_INCREF(args[kEntries]);
    Py_XSETREF(f_check, args[kEntries]);
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"bind", (PyCFunction)(void (*)(void))py_bind, METH_FASTCALL, nullptr},
    {"gemm", (PyCFunction)(void (*)(void))py_gemm, METH_FASTCALL, nullptr},
    {"conv2d_fwd", (PyCFunction)(void (*)(void))py_conv2d_fwd, METH_FASTCALL, nullptr},
    {"conv2d_winograd", (PyCFunction)(void (*)(void))py_conv2d_winograd, METH_FASTCALL, nullptr},
    {"quantize_i8", (PyCFunction)(void (*)(void))py_quantize_i8, METH_FASTCALL, nullptr},
    {"rmsnorm_i8", (PyCFunction)(void (*)(void))py_rmsnorm_i8, METH_FASTCALL, nullptr},
    {"gated_i8", (PyCFunction)(void (*)(void))py_gated_i8, METH_FASTCALL, nullptr},
    {"dequantize_i8", (PyCFunction)(void (*)(void))py_dequantize_i8, METH_FASTCALL, nullptr},
    {"gemm_i8", (PyCFunction)(void (*)(void))py_gemm_i8, METH_FASTCALL, nullptr},
    {"rope_qk", (PyCFunction)(void (*)(void))py_rope_qk, METH_FASTCALL, nullptr},
    {"rope_qk_backward", (PyCFunction)(void (*)(void))py_rope_qk_backward, METH_FASTCALL, nullptr},
    {"cache_append", (PyCFunction)(void (*)(void))py_cache_append, METH_FASTCALL, nullptr},
    {"attention_tree", (PyCFunction)(void (*)(void))py_attention_tree, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_pk_torch", "Native marshalling of the tensor calls.", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pk_torch(void)
{
    PyObject *m = PyModule_Create(&kModule);
    // the torch this was built for: binding.py takes no other
    if (m && PyModule_AddStringConstant(m, "torch_version", PK_TORCH_VERSION) < 0) Py_CLEAR(m);
    return m;
}
