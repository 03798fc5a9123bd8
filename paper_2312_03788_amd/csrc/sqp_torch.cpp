// Argument marshalling of the serving calls (GEMM, norms, activation smoothing, cache, attention) and of the calls that
// prepare a weight for torch tensors, in C++: a decode launch takes 5 to 15 us on the GPU, the same checks and
// the ctypes conversion in Python 11 us per GEMM call; the calls on a 1024 x 1024 weight take 9 to 14 us of
// host time in Python and 4 to 7 here.  Holds no arithmetic and no state but the addresses of the
// library's entry points, which the Python binding hands over (so that it always calls the library
// that the binding loaded).
//
// Every function returns the output tensor, or None for anything but the plain case (wrong type,
// device, layout or shape, tensor subclasses, a workspace that has to grow): nothing has been enqueued
// then, and the binding takes its general path, which reports the error.  Once the library has been
// called its code is the result: an error comes back as an integer, never as None, because the call
// may have been enqueued all the same (the status also carries errors of earlier work) and must not run
// twice.  Tensor methods may throw (nested tensors have no size in every dimension), so all of
// them are called inside a try block.  The library's
// calls run without the GIL, as under ctypes: a launch may have to wait for room in the queue.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_cuda_dispatch.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

namespace {

typedef int (*GemmFn)(int, int, int, int, const void *, const uint32_t *, const void *, const uint8_t *, void *, void *);
typedef size_t (*WorkspaceFn)(int, int, int, int);
typedef int (*ScratchGemmFn)(int, int, int, int, int, const void *, const uint32_t *, const void *, const uint8_t *, void *, void *, size_t, void *);
typedef int (*RmsnormFn)(int, int, const void *, const void *, float, void *, void *);
typedef int (*ApplyFn)(int, int, const void *, const float *, void *, void *);

typedef int (*ScalesFn)(int, int, int, float, const void *, const void *, float *, void *);
typedef int (*PackFn)(int, int, int, const void *, uint32_t *, void *, uint8_t *, void *);
typedef int (*UnpackFn)(int, int, int, const uint32_t *, const void *, const uint8_t *, void *, void *);
typedef int (*TransposeFn)(int, int, const void *, void *, void *);
typedef int (*InterleaveFn)(int, int, const void *, const void *, void *, void *);

typedef int (*AddNormFn)(int, int, const void *, const void *, const void *, float, void *, void *, void *);
typedef int (*AddNormQuantFn)(int, int, int, const void *, const void *, const void *, float, void *, float *, void *, void *);
typedef int (*CacheWriteFn)(int, int, int, int, int, int, int, const void *, long, const void *, long, const void *, long, const int *, const float *,
                            const int *, int, void *, void *, void *, void *, void *, void *);
typedef int (*CacheReadFn)(int, int, int, int, int, int, const int *, const void *, const void *, const void *, const void *, void *, void *, void *);
typedef int (*AttentionFn)(int, int, int, int, int, int, int, int, int, int, int, float, const void *, long, const void *, const void *, const void *,
                           const void *, const int *, long, const int *, const int *, void *, void *, size_t, void *);
typedef size_t (*AttentionScratchFn)(int, int, int, int, int, int, int);
typedef int (*MxQuantizeFn)(int, int, int, const void *, void *, uint8_t *, void *);
typedef int (*MxDequantizeFn)(int, int, int, const void *, const uint8_t *, void *, void *);
typedef int (*MxWeightFn)(int, int, const void *, void *, uint8_t *, void *);
typedef int (*MxGemmFn)(int, int, int, int, int, const void *, const uint8_t *, const void *, const uint8_t *, void *, void *, size_t, void *);
typedef size_t (*MxScratchFn)(int, int, int, int);
typedef int (*AddNormMxFn)(int, int, int, const void *, const void *, const void *, float, void *, uint8_t *, void *, void *);

GemmFn g_gemm[3];  // plain, fused activation, static scratch
WorkspaceFn g_workspace_bytes, g_scratch_bytes;
ScratchGemmFn g_gemm_scratch;
RmsnormFn g_rmsnorm;
ApplyFn g_apply[3];  // x / s and s * w per row of w, w / s per column
ScalesFn g_scales;
PackFn g_pack;
UnpackFn g_unpack;
TransposeFn g_transpose;
InterleaveFn g_interleave;
AddNormFn g_add_norm;
AddNormQuantFn g_add_norm_quant;
CacheWriteFn g_cache_write;
CacheReadFn g_cache_read;
AttentionFn g_attention;
AttentionScratchFn g_attention_scratch;
MxQuantizeFn g_mx_quantize;
MxDequantizeFn g_mx_dequantize;
MxWeightFn g_mx_weight;
MxGemmFn g_mx_gemm;
MxScratchFn g_mx_scratch;
AddNormMxFn g_add_norm_mx;

// The tensor behind an argument if it is a dense GPU tensor of this type on device `dev`, else null.  A
// subclass other than torch.nn.Parameter has semantics of its own (__torch_function__, the type of
// what torch.empty_like makes of it), with or without a dispatch key that tells.
const at::Tensor *plain(PyObject *o, at::ScalarType type, long dev)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.key_set().has(c10::DispatchKey::Python) || t.layout() != at::kStrided || !t.is_cuda()) return nullptr;
    if (t.scalar_type() != type || t.get_device() != dev || !t.is_contiguous()) return nullptr;
    return &t;
}

// A new tensor on the device of `like`.  Without dispatch modes, transforms, inference or grad modes that change the
// thread's dispatch keys the dispatcher ends at the GPU's own `empty`: that is called straight away then
// (0.7 us of a call of 4 to 5 instead of 0.8), unless a profiler or another observer records the operators.
at::Tensor fresh(at::IntArrayRef size, at::ScalarType type, const at::Tensor &like)
{
    const c10::impl::LocalDispatchKeySet tls = c10::impl::tls_local_dispatch_key_set();
    if (tls.included_ == c10::default_included_set && tls.excluded_ == c10::default_excluded_set && !at::hasCallbacks())
        return at::cuda::empty(size, type, at::kStrided, like.device(), false, c10::nullopt);
    return at::empty(size, like.options().dtype(type));
}

// `out` as given, or a new tensor like `like` with rows x cols elements (a given one is only taken
// if it has exactly that many).
bool output(PyObject *out, const at::Tensor &like, long rows, long cols, long dev, at::Tensor &y, at::ScalarType type = at::kHalf)
{
    if (out == Py_None) {
        y = fresh({rows, cols}, type, like);
        return true;
    }
    const at::Tensor *t = plain(out, type, dev);
    if (!t || t->numel() != rows * cols) return false;
    y = *t;
    return true;
}

PyObject *result(int rc, PyObject *out, const at::Tensor &y)
{
    if (rc != 0) return PyLong_FromLong(rc);
    if (out == Py_None) return THPVariable_Wrap(y);
    Py_INCREF(out);
    return out;
}

bool fits(long v) { return v > 0 && v <= INT_MAX; }

// gemm(which, x, packed, scales, zeros, group, out, device, stream, workspace bytes held)
PyObject *gemm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 10) Py_RETURN_NONE;
    const long which = PyLong_AsLong(a[0]), group = PyLong_AsLong(a[5]), dev = PyLong_AsLong(a[7]);
    void *stream = PyLong_AsVoidPtr(a[8]);
    const size_t held = PyLong_AsSize_t(a[9]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (which < 0 || which > 2 || !g_gemm[which]) Py_RETURN_NONE;
    try {
        const at::Tensor *x = plain(a[1], at::kHalf, dev), *packed = plain(a[2], at::kInt, dev);
        const at::Tensor *scales = plain(a[3], at::kHalf, dev), *zeros = plain(a[4], at::kByte, dev);
        if (!x || !packed || !scales || !zeros || x->dim() != 2 || packed->dim() != 2) Py_RETURN_NONE;
        const long M = x->size(0), K = x->size(1), N = packed->size(1);
        if (!fits(M) || !fits(K) || !fits(N) || !fits(group) || packed->size(0) * 8 != K) Py_RETURN_NONE;
        if (which != 2 && g_workspace_bytes((int)M, (int)N, (int)K, (int)group) > held) Py_RETURN_NONE;
        // scratch of this call alone: freed to the allocator's pool of this stream when the call returns, so
        // whatever takes it next is ordered behind the kernels (with `out` the general path looks
        // whether the caller may not allocate)
        const size_t own = which == 2 ? 0 : g_scratch_bytes((int)M, (int)N, (int)K, (int)group);
        if (own > 0 && a[6] != Py_None) Py_RETURN_NONE;
        at::Tensor y, scratch;
        if (!output(a[6], *x, M, which == 1 ? N / 2 : N, dev, y)) Py_RETURN_NONE;
        const void *xp = x->data_ptr(), *pp = packed->data_ptr(), *sp = scales->data_ptr(), *zp = zeros->data_ptr();
        void *yp = y.data_ptr();
        if (own > 0) scratch = fresh({(long)own}, at::kByte, *x);
        void *op = own > 0 ? scratch.data_ptr() : nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        if (own > 0)
            rc = g_gemm_scratch((int)M, (int)N, (int)K, (int)group, which, xp, (const uint32_t *)pp, sp, (const uint8_t *)zp, yp, op, own, stream);
        else
            rc = g_gemm[which]((int)M, (int)N, (int)K, (int)group, xp, (const uint32_t *)pp, sp, (const uint8_t *)zp, yp, stream);
        Py_END_ALLOW_THREADS
        return result(rc, a[6], y);
    } catch (...) {  // e.g. out of memory: the general path raises it as Python does
        Py_RETURN_NONE;
    }
}

// rmsnorm(x, gamma, eps, out, device, stream)
PyObject *rmsnorm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 6) Py_RETURN_NONE;
    const double eps = PyFloat_AsDouble(a[2]);
    const long dev = PyLong_AsLong(a[4]);
    void *stream = PyLong_AsVoidPtr(a[5]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    try {
        const at::Tensor *x = plain(a[0], at::kHalf, dev), *gamma = plain(a[1], at::kHalf, dev);
        if (!x || !gamma || x->dim() != 2 || !fits(x->size(0)) || !fits(x->size(1))) Py_RETURN_NONE;
        const long M = x->size(0), H = x->size(1);
        at::Tensor y;
        if (!output(a[3], *x, M, H, dev, y)) Py_RETURN_NONE;
        const void *xp = x->data_ptr(), *gp = gamma->data_ptr();
        void *yp = y.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_rmsnorm((int)M, (int)H, xp, gp, (float)eps, yp, stream);
        Py_END_ALLOW_THREADS
        return result(rc, a[3], y);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// The last two arguments of the calls below; false: not whole numbers.
bool place(PyObject *const *a, Py_ssize_t n, long &dev, void *&stream)
{
    dev = PyLong_AsLong(a[n - 2]);
    stream = PyLong_AsVoidPtr(a[n - 1]);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}

// apply(which, x, s, out, device, stream): x / s (0), s * x (1: per row), x / s (2: per column)
PyObject *apply(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 6 || !place(a, n, dev, stream)) Py_RETURN_NONE;
    const long which = PyLong_AsLong(a[0]);
    if (which < 0 || which > 2 || !g_apply[which]) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    try {
        const at::Tensor *x = plain(a[1], at::kHalf, dev), *s = plain(a[2], at::kFloat, dev);
        if (!x || !s || x->dim() != 2 || !fits(x->size(0)) || !fits(x->size(1))) Py_RETURN_NONE;
        const long rows = x->size(0), cols = x->size(1);
        at::Tensor y;
        if (!output(a[3], *x, rows, cols, dev, y)) Py_RETURN_NONE;
        const void *xp = x->data_ptr(), *sp = s->data_ptr();
        void *yp = y.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_apply[which]((int)rows, (int)cols, xp, (const float *)sp, yp, stream);
        Py_END_ALLOW_THREADS
        return result(rc, a[3], y);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// smooth_scales(x_cal, w, alpha, out, device, stream)
PyObject *smooth_scales(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 6 || !g_scales || !place(a, n, dev, stream)) Py_RETURN_NONE;
    const double alpha = PyFloat_AsDouble(a[2]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    try {
        const at::Tensor *x = plain(a[0], at::kHalf, dev), *w = plain(a[1], at::kHalf, dev);
        if (!x || !w || x->dim() != 2 || w->dim() != 2 || x->size(1) != w->size(0)) Py_RETURN_NONE;
        const long T = x->size(0), K = x->size(1), N = w->size(1);
        if (!fits(T) || !fits(K) || !fits(N)) Py_RETURN_NONE;
        at::Tensor s;
        if (a[3] == Py_None) s = fresh({K}, at::kFloat, *w);
        else if (!output(a[3], *w, K, 1, dev, s, at::kFloat)) Py_RETURN_NONE;
        const void *xp = x->data_ptr(), *wp = w->data_ptr();
        void *sp = s.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_scales((int)T, (int)K, (int)N, (float)alpha, xp, wp, (float *)sp, stream);
        Py_END_ALLOW_THREADS
        return result(rc, a[3], s);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// quantize_pack(w, group, device, stream): new (packed, scales, zeros)
PyObject *quantize_pack(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 4 || !g_pack || !place(a, n, dev, stream)) Py_RETURN_NONE;
    const long group = PyLong_AsLong(a[1]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    try {
        const at::Tensor *w = plain(a[0], at::kHalf, dev);
        if (!w || w->dim() != 2 || !fits(group)) Py_RETURN_NONE;
        const long K = w->size(0), N = w->size(1);
        if (!fits(K) || !fits(N) || K % group || K % 8) Py_RETURN_NONE;
        const at::Tensor packed = fresh({K / 8, N}, at::kInt, *w), scales = fresh({K / group, N}, at::kHalf, *w),
                         zeros = fresh({K / group, N}, at::kByte, *w);
        const void *wp = w->data_ptr();
        void *pp = packed.data_ptr(), *sp = scales.data_ptr(), *zp = zeros.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_pack((int)N, (int)K, (int)group, wp, (uint32_t *)pp, sp, (uint8_t *)zp, stream);
        Py_END_ALLOW_THREADS
        if (rc != 0) return PyLong_FromLong(rc);
        return Py_BuildValue("(NNN)", THPVariable_Wrap(packed), THPVariable_Wrap(scales), THPVariable_Wrap(zeros));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// dequantize(packed, scales, zeros, group, out, device, stream)
PyObject *dequantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 7 || !g_unpack || !place(a, n, dev, stream)) Py_RETURN_NONE;
    const long group = PyLong_AsLong(a[3]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    try {
        const at::Tensor *packed = plain(a[0], at::kInt, dev), *scales = plain(a[1], at::kHalf, dev), *zeros = plain(a[2], at::kByte, dev);
        if (!packed || !scales || !zeros || packed->dim() != 2 || !fits(group)) Py_RETURN_NONE;
        const long K = packed->size(0) * 8, N = packed->size(1);
        if (!fits(K) || !fits(N)) Py_RETURN_NONE;
        at::Tensor y;
        if (!output(a[4], *scales, K, N, dev, y)) Py_RETURN_NONE;
        const void *pp = packed->data_ptr(), *sp = scales->data_ptr(), *zp = zeros->data_ptr();
        void *yp = y.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_unpack((int)N, (int)K, (int)group, (const uint32_t *)pp, sp, (const uint8_t *)zp, yp, stream);
        Py_END_ALLOW_THREADS
        return result(rc, a[4], y);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// transpose_nk(w_nk, out, device, stream)
PyObject *transpose_nk(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 4 || !g_transpose || !place(a, n, dev, stream)) Py_RETURN_NONE;
    try {
        const at::Tensor *w = plain(a[0], at::kHalf, dev);
        if (!w || w->dim() != 2 || !fits(w->size(0)) || !fits(w->size(1))) Py_RETURN_NONE;
        const long N = w->size(0), K = w->size(1);
        at::Tensor y;
        if (!output(a[1], *w, K, N, dev, y)) Py_RETURN_NONE;
        const void *wp = w->data_ptr();
        void *yp = y.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_transpose((int)N, (int)K, wp, yp, stream);
        Py_END_ALLOW_THREADS
        return result(rc, a[1], y);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// interleave_gate_up(w_gate, w_up, out, device, stream): two tensors of one shape
PyObject *interleave_gate_up(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 5 || !g_interleave || !place(a, n, dev, stream)) Py_RETURN_NONE;
    try {
        const at::Tensor *gate = plain(a[0], at::kHalf, dev), *up = plain(a[1], at::kHalf, dev);
        if (!gate || !up || gate->dim() != 2 || !up->sizes().equals(gate->sizes())) Py_RETURN_NONE;
        const long K = gate->size(0), I = gate->size(1);
        if (!fits(K) || !fits(2 * I)) Py_RETURN_NONE;
        at::Tensor y;
        if (!output(a[2], *gate, K, 2 * I, dev, y)) Py_RETURN_NONE;
        const void *gp = gate->data_ptr(), *upp = up->data_ptr();
        void *yp = y.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_interleave((int)K, (int)I, gp, upp, yp, stream);
        Py_END_ALLOW_THREADS
        return result(rc, a[2], y);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// bind(addresses of sqp_w4a16_gemm, _silu_mul, _static, _workspace_bytes, sqp_rmsnorm, sqp_smooth_apply_x,
//      sqp_w4a16_gemm_scratch, _scratch_bytes)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[8];
    if (n != 8) {
        PyErr_SetString(PyExc_TypeError, "bind takes eight addresses");
        return nullptr;
    }
    for (int i = 0; i < 8; i++) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    for (int i = 0; i < 3; i++) g_gemm[i] = (GemmFn)p[i];
    g_workspace_bytes = (WorkspaceFn)p[3];
    g_rmsnorm = (RmsnormFn)p[4];
    g_apply[0] = (ApplyFn)p[5];
    g_gemm_scratch = (ScratchGemmFn)p[6];
    g_scratch_bytes = (WorkspaceFn)p[7];
    Py_RETURN_NONE;
}

// bind_preparation(addresses of sqp_smooth_apply_w, sqp_scale_columns, sqp_smooth_scales, sqp_quantize_pack, sqp_dequantize,
//      sqp_transpose_nk, sqp_interleave_gate_up)
PyObject *bind_preparation(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[7];
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "bind_preparation takes seven addresses");
        return nullptr;
    }
    for (int i = 0; i < 7; i++) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    g_apply[1] = (ApplyFn)p[0];
    g_apply[2] = (ApplyFn)p[1];
    g_scales = (ScalesFn)p[2];
    g_pack = (PackFn)p[3];
    g_unpack = (UnpackFn)p[4];
    g_transpose = (TransposeFn)p[5];
    g_interleave = (InterleaveFn)p[6];
    Py_RETURN_NONE;
}

// add_rmsnorm(type, x, residual, gamma, eps, out, sum out, device, stream): new (y, sum) or (codes, scales, sum)
PyObject *add_rmsnorm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 9 || !g_add_norm || !place(a, n, dev, stream)) Py_RETURN_NONE;
    const long type = PyLong_AsLong(a[0]);
    const double eps = PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (type < 0 || type > 2 || (type && a[5] != Py_None)) Py_RETURN_NONE;
    try {
        const at::Tensor *x = plain(a[1], at::kHalf, dev), *residual = plain(a[2], at::kHalf, dev), *gamma = plain(a[3], at::kHalf, dev);
        if (!x || !residual || !gamma || x->dim() != 2 || !residual->sizes().equals(x->sizes()) || gamma->dim() != 1 || gamma->size(0) != x->size(1)) Py_RETURN_NONE;
        const long M = x->size(0), H = x->size(1);
        if (!fits(M) || !fits(H)) Py_RETURN_NONE;
        at::Tensor y, sum, scales;
        for (int i = 5; i < 7; i++) {  // (given outputs have the shape of x)
            const at::Tensor *t = a[i] == Py_None ? x : plain(a[i], at::kHalf, dev);
            if (!t || !t->sizes().equals(x->sizes())) Py_RETURN_NONE;
            (i == 5 ? y : sum) = a[i] == Py_None ? fresh({M, H}, i == 6 || type == 0 ? at::kHalf : type == 1 ? at::kChar : at::kFloat8_e4m3fn, *x) : *t;
        }
        if (type) scales = fresh({M}, at::kFloat, *x);
        const void *xp = x->data_ptr(), *rp = residual->data_ptr(), *gp = gamma->data_ptr();
        void *yp = y.data_ptr(), *sp = sum.data_ptr(), *cp = type ? scales.data_ptr() : nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        if (type) rc = g_add_norm_quant((int)M, (int)H, (int)type, xp, rp, gp, (float)eps, yp, (float *)cp, sp, stream);
        else rc = g_add_norm((int)M, (int)H, xp, rp, gp, (float)eps, yp, sp, stream);
        Py_END_ALLOW_THREADS
        if (rc != 0) return PyLong_FromLong(rc);
        PyObject *yo = a[5], *so = a[6];
        if (yo == Py_None) yo = THPVariable_Wrap(y);
        else Py_INCREF(yo);
        if (so == Py_None) so = THPVariable_Wrap(sum);
        else Py_INCREF(so);
        return type ? Py_BuildValue("(NNN)", yo, THPVariable_Wrap(scales), so) : Py_BuildValue("(NN)", yo, so);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// A tensor [tokens, heads, D] in fp16 whose tokens may lie apart, and the distance between them; else null.
const at::Tensor *tokens(PyObject *o, long dev, long &step)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.key_set().has(c10::DispatchKey::Python) || t.layout() != at::kStrided || !t.is_cuda()) return nullptr;
    if (t.scalar_type() != at::kHalf || t.get_device() != dev || t.dim() != 3 || t.size(0) <= 0 || t.size(0) > INT_MAX) return nullptr;
    if (t.stride(2) != 1 || (t.size(1) > 1 && t.stride(1) != t.size(2))) return nullptr;
    step = t.size(0) > 1 ? t.stride(0) : t.size(1) * t.size(2);
    return &t;
}

struct Cache {
    const at::Tensor *k, *v, *k_scales, *v_scales;
    int pages, kv_heads, page, D, type;
    void *kp, *vp, *ksp, *vsp;
};

// The cache of four arguments: k_cache, v_cache, k_scales, v_scales.
bool cache(PyObject *const *a, long dev, Cache &c)
{
    if (!THPVariable_CheckExact(a[0])) return false;
    const at::Tensor &t = THPVariable_Unpack(a[0]);
    if (!t.defined()) return false;
    const at::ScalarType type = t.scalar_type();
    c.type = type == at::kHalf ? 0 : type == at::kChar ? 1 : type == at::kFloat8_e4m3fn ? 2 : type == at::kByte ? 4 : -1;  // (kByte: e2m1, two to a byte)
    if (c.type < 0) return false;
    c.k = plain(a[0], type, dev);
    c.v = plain(a[1], type, dev);
    if (!c.k || !c.v || c.k->dim() != 4 || !c.v->sizes().equals(c.k->sizes())) return false;
    for (int i = 0; i < 4; i++)
        if (!fits(c.k->size(i))) return false;
    c.pages = (int)c.k->size(0); c.kv_heads = (int)c.k->size(1); c.page = (int)c.k->size(2); c.D = (int)c.k->size(3);
    if (c.type == 4) {
        if (c.D > 64) return false;
        c.D *= 2;
    }
    c.kp = c.k->data_ptr();
    c.vp = c.v->data_ptr();
    c.ksp = c.vsp = nullptr;
    if (c.type == 0) return a[2] == Py_None && a[3] == Py_None;
    const at::ScalarType scale = c.type == 4 ? at::kByte : at::kFloat;  // e2m1: a byte per block of 32, else one scale per token and head
    const long dims = c.type == 4 ? 4 : 3;
    c.k_scales = plain(a[2], scale, dev);
    c.v_scales = plain(a[3], scale, dev);
    if (!c.k_scales || !c.v_scales || c.k_scales->dim() != dims || !c.v_scales->sizes().equals(c.k_scales->sizes())) return false;
    if (!c.k_scales->sizes().slice(0, 3).equals(c.k->sizes().slice(0, 3)) || (dims == 4 && c.k_scales->size(3) != c.D / 32)) return false;
    c.ksp = c.k_scales->data_ptr();
    c.vsp = c.v_scales->data_ptr();
    return true;
}

bool is_tokens(const at::Tensor *t, long T, long heads, long D) { return t && t->size(0) == T && t->size(1) == heads && t->size(2) == D; }

// kv_cache_write(k, v, slots, k_cache, v_cache, k_scales, v_scales, q, cos_sin, positions, out, device, stream): the queries, or
// True where there are none
PyObject *kv_cache_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 13 || !g_cache_write || !place(a, n, dev, stream)) Py_RETURN_NONE;
    try {
        Cache c;
        if (!cache(a + 3, dev, c)) Py_RETURN_NONE;
        long k_step, v_step, q_step = 0;
        const at::Tensor *k = tokens(a[0], dev, k_step), *v = tokens(a[1], dev, v_step), *slots = plain(a[2], at::kInt, dev);
        if (!k || !is_tokens(k, k->size(0), c.kv_heads, c.D) || !is_tokens(v, k->size(0), c.kv_heads, c.D)) Py_RETURN_NONE;
        const long T = k->size(0);
        if (!slots || slots->dim() != 1 || slots->size(0) != T) Py_RETURN_NONE;
        const at::Tensor *q = nullptr, *cos_sin = nullptr, *positions = nullptr;
        at::Tensor y;
        if (a[7] != Py_None) {
            q = tokens(a[7], dev, q_step);
            if (!q || !is_tokens(q, T, q->size(1), c.D) || !fits(q->size(1))) Py_RETURN_NONE;
            if (a[10] == Py_None) {
                y = fresh({T, q->size(1), c.D}, at::kHalf, *q);
            } else {
                const at::Tensor *o = plain(a[10], at::kHalf, dev);
                if (!o || !o->sizes().equals(q->sizes())) Py_RETURN_NONE;
                y = *o;
            }
        }
        if (a[8] != Py_None) {
            cos_sin = plain(a[8], at::kFloat, dev);
            positions = plain(a[9], at::kInt, dev);
            if (!cos_sin || cos_sin->dim() != 2 || cos_sin->size(1) != c.D || !fits(cos_sin->size(0))) Py_RETURN_NONE;
            if (!positions || positions->dim() != 1 || positions->size(0) != T) Py_RETURN_NONE;
        }
        const void *qp = q ? q->data_ptr() : nullptr, *kp = k->data_ptr(), *vp = v->data_ptr();
        const int *sp = (const int *)slots->data_ptr(), *pp = positions ? (const int *)positions->data_ptr() : nullptr;
        const float *cp = cos_sin ? (const float *)cos_sin->data_ptr() : nullptr;
        const int heads = q ? (int)q->size(1) : 0, n_positions = cos_sin ? (int)cos_sin->size(0) : 0;
        void *yp = q ? y.data_ptr() : nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_cache_write((int)T, heads, c.kv_heads, c.D, c.type, c.page, c.pages, qp, q_step, kp, k_step, vp, v_step, sp, cp, pp, n_positions, c.kp, c.vp,
                           c.ksp, c.vsp, yp, stream);
        Py_END_ALLOW_THREADS
        if (rc == 0 && !q) Py_RETURN_TRUE;
        return result(rc, q ? a[10] : Py_None, y);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// kv_cache_read(slots, k_cache, v_cache, k_scales, v_scales, device, stream): new (k, v)
PyObject *kv_cache_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 7 || !g_cache_read || !place(a, n, dev, stream)) Py_RETURN_NONE;
    try {
        Cache c;
        const at::Tensor *slots = plain(a[0], at::kInt, dev);
        if (!slots || slots->dim() != 1 || !fits(slots->size(0)) || !cache(a + 1, dev, c)) Py_RETURN_NONE;
        const long T = slots->size(0);
        const at::Tensor k = fresh({T, c.kv_heads, c.D}, at::kHalf, *slots), v = fresh({T, c.kv_heads, c.D}, at::kHalf, *slots);
        const int *sp = (const int *)slots->data_ptr();
        void *kp = k.data_ptr(), *vp = v.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_cache_read((int)T, c.kv_heads, c.D, c.type, c.page, c.pages, sp, c.kp, c.vp, c.ksp, c.vsp, kp, vp, stream);
        Py_END_ALLOW_THREADS
        if (rc != 0) return PyLong_FromLong(rc);
        return Py_BuildValue("(NN)", THPVariable_Wrap(k), THPVariable_Wrap(v));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// paged_attention(q, k_cache, v_cache, page_table, seq_lens, q_starts, k_scales, v_scales, max_q, max_len, scale, out, device, stream)
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 14 || !g_attention || !place(a, n, dev, stream)) Py_RETURN_NONE;
    const long max_q = a[5] == Py_None ? 1 : a[8] == Py_None ? 0 : PyLong_AsLong(a[8]), max_len = a[9] == Py_None ? 0 : PyLong_AsLong(a[9]);
    const double given = a[10] == Py_None ? 0.0 : PyFloat_AsDouble(a[10]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (max_q < 0 || max_q > INT_MAX || max_len < 0 || max_len > INT_MAX) Py_RETURN_NONE;
    try {
        Cache c;
        PyObject *const four[4] = {a[1], a[2], a[6], a[7]};
        if (!cache(four, dev, c)) Py_RETURN_NONE;
        long q_step;
        const at::Tensor *q = tokens(a[0], dev, q_step), *lens = plain(a[4], at::kInt, dev), *starts = nullptr;
        if (!q || q->size(2) != c.D || !fits(q->size(1)) || q->size(1) % c.kv_heads || !lens || lens->dim() != 1 || !THPVariable_CheckExact(a[3])) Py_RETURN_NONE;
        const at::Tensor &table = THPVariable_Unpack(a[3]);
        if (!table.defined() || table.key_set().has(c10::DispatchKey::Python) || table.layout() != at::kStrided || !table.is_cuda()) Py_RETURN_NONE;
        if (table.scalar_type() != at::kInt || table.get_device() != dev || table.dim() != 2) Py_RETURN_NONE;
        const long T = q->size(0), heads = q->size(1), B = table.size(0), width = table.size(1);
        if (!fits(B) || !fits(width) || lens->size(0) != B || (width > 1 && table.stride(1) != 1)) Py_RETURN_NONE;
        if (a[5] != Py_None) {
            starts = plain(a[5], at::kInt, dev);
            if (!starts || starts->dim() != 1 || starts->size(0) != B + 1) Py_RETURN_NONE;
        } else if (T != B) {
            Py_RETURN_NONE;
        }
        const long reach = width * c.page;
        const size_t bytes = g_attention_scratch((int)T, (int)B, (int)heads, c.kv_heads, c.D, (int)max_q, (int)(max_len ? max_len : reach > INT_MAX ? INT_MAX : reach));
        if (bytes > 0 && a[11] != Py_None) Py_RETURN_NONE;  // (the general path looks whether the caller may not allocate)
        at::Tensor y, scratch;
        if (a[11] == Py_None) {
            y = fresh({T, heads, c.D}, at::kHalf, *q);
        } else {
            const at::Tensor *o = plain(a[11], at::kHalf, dev);
            if (!o || !o->sizes().equals(q->sizes())) Py_RETURN_NONE;
            y = *o;
        }
        if (bytes > 0) scratch = fresh({(long)bytes}, at::kByte, *q);  // (dropped on return: whatever takes it next is ordered behind the kernels)
        const void *qp = q->data_ptr();
        const int *tp = (const int *)table.data_ptr(), *lp = (const int *)lens->data_ptr(), *sp = starts ? (const int *)starts->data_ptr() : nullptr;
        const long t_step = B > 1 ? table.stride(0) : width;
        void *yp = y.data_ptr(), *wp = bytes > 0 ? scratch.data_ptr() : nullptr;
        const float scale = a[10] == Py_None ? (c.D == 128 ? 0.08838834764831845f : 0.125f) : (float)given;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_attention((int)T, (int)B, (int)heads, c.kv_heads, c.D, c.type, c.page, c.pages, (int)width, (int)max_q, (int)max_len, scale, qp, q_step, c.kp,
                         c.vp, c.ksp, c.vsp, tp, t_step, lp, sp, yp, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        return result(rc, a[11], y);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// bind_layer(addresses of sqp_add_rmsnorm, _quant, sqp_kv_cache_write, _read, sqp_paged_attention, _scratch_bytes)
PyObject *bind_layer(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[6];
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "bind_layer takes six addresses");
        return nullptr;
    }
    for (int i = 0; i < 6; i++) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    g_add_norm = (AddNormFn)p[0];
    g_add_norm_quant = (AddNormQuantFn)p[1];
    g_cache_write = (CacheWriteFn)p[2];
    g_cache_read = (CacheReadFn)p[3];
    g_attention = (AttentionFn)p[4];
    g_attention_scratch = (AttentionScratchFn)p[5];
    Py_RETURN_NONE;
}

// The values per row of codes, 0 if they are none.
const at::Tensor *mx_rows(PyObject *codes, PyObject *scales, long dev, const at::Tensor *&s, long &R, long &K, int &type)
{
    if (!THPVariable_CheckExact(codes)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(codes);
    if (!t.defined()) return nullptr;
    type = t.scalar_type() == at::kByte ? 4 : t.scalar_type() == at::kFloat8_e4m3fn ? 2 : 0;
    const at::Tensor *c = type ? plain(codes, t.scalar_type(), dev) : nullptr;
    s = plain(scales, at::kByte, dev);
    if (!c || !s || c->dim() != 2 || s->dim() != 2) return nullptr;
    R = c->size(0);
    K = c->size(1) * (type == 4 ? 2 : 1);
    return fits(R) && fits(K) && K % 32 == 0 && s->size(0) == R && s->size(1) == K / 32 ? c : nullptr;
}

// mx_quantize(type, x, device, stream): new (codes, scales)
PyObject *mx_quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 4 || !g_mx_quantize || !place(a, n, dev, stream)) Py_RETURN_NONE;
    const long type = PyLong_AsLong(a[0]);
    if (type != 4 && type != 2) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    try {
        const at::Tensor *x = plain(a[1], at::kHalf, dev);
        if (!x || x->dim() != 2 || !fits(x->size(0)) || !fits(x->size(1)) || x->size(1) % 32) Py_RETURN_NONE;
        const long R = x->size(0), K = x->size(1);
        const at::Tensor codes = type == 4 ? fresh({R, K / 2}, at::kByte, *x) : fresh({R, K}, at::kFloat8_e4m3fn, *x), scales = fresh({R, K / 32}, at::kByte, *x);
        const void *xp = x->data_ptr();
        void *cp = codes.data_ptr();
        uint8_t *sp = (uint8_t *)scales.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_mx_quantize((int)R, (int)K, (int)type, xp, cp, sp, stream);
        Py_END_ALLOW_THREADS
        if (rc != 0) return PyLong_FromLong(rc);
        return Py_BuildValue("(NN)", THPVariable_Wrap(codes), THPVariable_Wrap(scales));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// mx_quantize_weight(w, device, stream): new (codes, scales)
PyObject *mx_quantize_weight(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 3 || !g_mx_weight || !place(a, n, dev, stream)) Py_RETURN_NONE;
    try {
        const at::Tensor *w = plain(a[0], at::kHalf, dev);
        if (!w || w->dim() != 2 || !fits(w->size(0)) || !fits(w->size(1)) || w->size(0) % 32) Py_RETURN_NONE;
        const long K = w->size(0), N = w->size(1);
        const at::Tensor codes = fresh({N, K / 2}, at::kByte, *w), scales = fresh({N, K / 32}, at::kByte, *w);
        const void *wp = w->data_ptr();
        void *cp = codes.data_ptr();
        uint8_t *sp = (uint8_t *)scales.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_mx_weight((int)N, (int)K, wp, cp, sp, stream);
        Py_END_ALLOW_THREADS
        if (rc != 0) return PyLong_FromLong(rc);
        return Py_BuildValue("(NN)", THPVariable_Wrap(codes), THPVariable_Wrap(scales));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// mx_dequantize(codes, scales, device, stream): new x
PyObject *mx_dequantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 4 || !g_mx_dequantize || !place(a, n, dev, stream)) Py_RETURN_NONE;
    try {
        const at::Tensor *scales;
        long R, K;
        int type;
        const at::Tensor *codes = mx_rows(a[0], a[1], dev, scales, R, K, type);
        if (!codes) Py_RETURN_NONE;
        const at::Tensor x = fresh({R, K}, at::kHalf, *codes);
        const void *cp = codes->data_ptr();
        const uint8_t *sp = (const uint8_t *)scales->data_ptr();
        void *xp = x.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_mx_dequantize((int)R, (int)K, type, cp, sp, xp, stream);
        Py_END_ALLOW_THREADS
        return result(rc, Py_None, x);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// mx_gemm(silu, x, x scales, w, w scales, out, device, stream)
PyObject *mx_gemm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 8 || !g_mx_gemm || !place(a, n, dev, stream)) Py_RETURN_NONE;
    const long silu = PyLong_AsLong(a[0]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    try {
        const at::Tensor *xs, *ws;
        long M, N, K, K2;
        int type, w_type;
        const at::Tensor *x = mx_rows(a[1], a[2], dev, xs, M, K, type), *w = mx_rows(a[3], a[4], dev, ws, N, K2, w_type);
        if (!x || !w || w_type != 4 || K != K2) Py_RETURN_NONE;
        const size_t bytes = g_mx_scratch((int)M, (int)N, (int)K, type);
        if (bytes > 0 && a[5] != Py_None) Py_RETURN_NONE;  // (the general path looks whether the caller may not allocate)
        const long cols = silu ? N / 2 : N;
        at::Tensor y, scratch;
        if (a[5] == Py_None) {
            y = fresh({M, cols}, at::kHalf, *x);
        } else {
            const at::Tensor *o = plain(a[5], at::kHalf, dev);
            if (!o || o->dim() != 2 || o->size(0) != M || o->size(1) != cols) Py_RETURN_NONE;
            y = *o;
        }
        if (bytes > 0) scratch = fresh({(long)bytes}, at::kByte, *x);  // (dropped on return: whatever takes it next is ordered behind the kernels)
        const void *xp = x->data_ptr(), *wp = w->data_ptr();
        const uint8_t *xsp = (const uint8_t *)xs->data_ptr(), *wsp = (const uint8_t *)ws->data_ptr();
        void *yp = y.data_ptr(), *sp = bytes > 0 ? scratch.data_ptr() : nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_mx_gemm((int)M, (int)N, (int)K, type, (int)silu, xp, xsp, wp, wsp, yp, sp, bytes, stream);
        Py_END_ALLOW_THREADS
        return result(rc, a[5], y);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// add_rmsnorm_mx(type, x, residual, gamma, eps, sum out, device, stream): new (codes, scales), and the sum
PyObject *add_rmsnorm_mx(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    long dev;
    void *stream;
    if (n != 8 || !g_add_norm_mx || !place(a, n, dev, stream)) Py_RETURN_NONE;
    const long type = PyLong_AsLong(a[0]);
    const double eps = PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred() || (type != 4 && type != 2)) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    try {
        const at::Tensor *x = plain(a[1], at::kHalf, dev), *residual = plain(a[2], at::kHalf, dev), *gamma = plain(a[3], at::kHalf, dev);
        if (!x || !residual || !gamma || x->dim() != 2 || !residual->sizes().equals(x->sizes()) || gamma->dim() != 1 || gamma->size(0) != x->size(1)) Py_RETURN_NONE;
        const long M = x->size(0), H = x->size(1);
        if (!fits(M) || !fits(H) || H % 32) Py_RETURN_NONE;
        at::Tensor sum;
        if (a[5] == Py_None) {
            sum = fresh({M, H}, at::kHalf, *x);
        } else {
            const at::Tensor *t = plain(a[5], at::kHalf, dev);
            if (!t || !t->sizes().equals(x->sizes())) Py_RETURN_NONE;
            sum = *t;
        }
        const at::Tensor codes = type == 4 ? fresh({M, H / 2}, at::kByte, *x) : fresh({M, H}, at::kFloat8_e4m3fn, *x), scales = fresh({M, H / 32}, at::kByte, *x);
        const void *xp = x->data_ptr(), *rp = residual->data_ptr(), *gp = gamma->data_ptr();
        void *cp = codes.data_ptr(), *sp = sum.data_ptr();
        uint8_t *bp = (uint8_t *)scales.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_add_norm_mx((int)M, (int)H, (int)type, xp, rp, gp, (float)eps, cp, bp, sp, stream);
        Py_END_ALLOW_THREADS
        if (rc != 0) return PyLong_FromLong(rc);
        PyObject *so = a[5];
        if (so == Py_None) so = THPVariable_Wrap(sum);
        else Py_INCREF(so);
        return Py_BuildValue("(NNN)", THPVariable_Wrap(codes), THPVariable_Wrap(scales), so);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// bind_mx(addresses of sqp_mx_quantize, _dequantize, _quantize_weight, sqp_mx_gemm, _scratch_bytes, sqp_add_rmsnorm_mx)
PyObject *bind_mx(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[6];
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "bind_mx takes six addresses");
        return nullptr;
    }
    for (int i = 0; i < 6; i++) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    g_mx_quantize = (MxQuantizeFn)p[0];
    g_mx_dequantize = (MxDequantizeFn)p[1];
    g_mx_weight = (MxWeightFn)p[2];
    g_mx_gemm = (MxGemmFn)p[3];
    g_mx_scratch = (MxScratchFn)p[4];
    g_add_norm_mx = (AddNormMxFn)p[5];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind_mx", (PyCFunction)(void (*)(void))bind_mx, METH_FASTCALL, nullptr},
    {"mx_quantize", (PyCFunction)(void (*)(void))mx_quantize, METH_FASTCALL, nullptr},
    {"mx_quantize_weight", (PyCFunction)(void (*)(void))mx_quantize_weight, METH_FASTCALL, nullptr},
    {"mx_dequantize", (PyCFunction)(void (*)(void))mx_dequantize, METH_FASTCALL, nullptr},
    {"mx_gemm", (PyCFunction)(void (*)(void))mx_gemm, METH_FASTCALL, nullptr},
    {"add_rmsnorm_mx", (PyCFunction)(void (*)(void))add_rmsnorm_mx, METH_FASTCALL, nullptr},
    {"bind_layer", (PyCFunction)(void (*)(void))bind_layer, METH_FASTCALL, nullptr},
    {"add_rmsnorm", (PyCFunction)(void (*)(void))add_rmsnorm, METH_FASTCALL, nullptr},
    {"kv_cache_write", (PyCFunction)(void (*)(void))kv_cache_write, METH_FASTCALL, nullptr},
    {"kv_cache_read", (PyCFunction)(void (*)(void))kv_cache_read, METH_FASTCALL, nullptr},
    {"paged_attention", (PyCFunction)(void (*)(void))paged_attention, METH_FASTCALL, nullptr},
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {"gemm", (PyCFunction)(void (*)(void))gemm, METH_FASTCALL, nullptr},
    {"rmsnorm", (PyCFunction)(void (*)(void))rmsnorm, METH_FASTCALL, nullptr},
    {"bind_preparation", (PyCFunction)(void (*)(void))bind_preparation, METH_FASTCALL, nullptr},
    {"apply", (PyCFunction)(void (*)(void))apply, METH_FASTCALL, nullptr},
    {"smooth_scales", (PyCFunction)(void (*)(void))smooth_scales, METH_FASTCALL, nullptr},
    {"quantize_pack", (PyCFunction)(void (*)(void))quantize_pack, METH_FASTCALL, nullptr},
    {"dequantize", (PyCFunction)(void (*)(void))dequantize, METH_FASTCALL, nullptr},
    {"transpose_nk", (PyCFunction)(void (*)(void))transpose_nk, METH_FASTCALL, nullptr},
    {"interleave_gate_up", (PyCFunction)(void (*)(void))interleave_gate_up, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sqp_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__sqp_torch() { return PyModule_Create(&module); }
