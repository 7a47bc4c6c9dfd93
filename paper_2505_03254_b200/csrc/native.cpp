// CPython entry points of the calls a program makes per layer or per step.
//
// A small layer runs in a few microseconds, less than ctypes needs to marshal its arguments (measured
// on the benchmark's host: 9.5 us per call through ctypes, of which 2.2 us are the launch).  These
// functions read the tensors' pointers, types and sizes straight from the tensor objects, ask for the
// current stream once, release the interpreter lock around the library call and return its status.
// They take positional arguments only; binding.py holds the documented signatures, the optional
// allocations and the exceptions for statuses.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "prom.h"

namespace {

// What a bad argument raises; caught at the boundary of every entry point.
struct ArgError {};

[[noreturn]] void fail(PyObject *type, const char *fmt, const char *name, const char *detail = "")
{
    PyErr_Format(type, fmt, name, detail);
    throw ArgError();
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s must be a tensor", name);
    return THPVariable_Unpack(o);
}

const char *dtype_name(at::ScalarType t)
{
    switch (t) {
    case at::kChar: return "torch.int8";
    case at::kByte: return "torch.uint8";
    case at::kInt: return "torch.int32";
    case at::kBFloat16: return "torch.bfloat16";
    case at::kHalf: return "torch.float16";
    default: return "torch.float32";
    }
}

// A contiguous CUDA tensor of the given type.
const at::Tensor &dev(PyObject *o, at::ScalarType t, const char *name)
{
    const at::Tensor &x = tensor(o, name);
    if (!x.is_cuda()) fail(PyExc_ValueError, "%s must be a CUDA tensor", name);
    if (x.scalar_type() != t || !x.is_contiguous())
        fail(PyExc_ValueError, "%s must be contiguous %s", name, dtype_name(t));
    return x;
}

template <class T> T *ptr(const at::Tensor &t) { return static_cast<T *>(t.data_ptr()); }

void dims(const at::Tensor &t, int64_t n, const char *name)
{
    if (t.dim() != n) {
        PyErr_Format(PyExc_ValueError, "%s must have %d dimensions, not %d", name, (int)n, (int)t.dim());
        throw ArgError();
    }
}

long long integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw ArgError();
    return v;
}

int small_int(PyObject *o)
{
    const long long v = integer(o);
    if (v != (int)v) {
        PyErr_SetString(PyExc_OverflowError, "integer argument out of range");
        throw ArgError();
    }
    return (int)v;
}

// A stream handle, or None for the current stream of the current device.
void *stream(PyObject *o)
{
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw ArgError();
    return p;
}

// The binding's ctypes structures, told by it once (register_types).
PyObject *requant_type, *layer_type, *job_type;

// A structure of the given type, or an array of them.
void structure(PyObject *o, PyObject *type, const char *name)
{
    if ((PyObject *)Py_TYPE(o) == type) return;
    static PyObject *const attr = PyUnicode_InternFromString("_type_");
    PyObject *element = PyObject_GetAttr((PyObject *)Py_TYPE(o), attr);       // of an array type
    if (!element) PyErr_Clear();
    const bool ok = element == type || (type && PyObject_IsInstance(o, type) == 1);
    Py_XDECREF(element);
    if (!ok) {
        PyErr_Clear();
        fail(PyExc_TypeError, "%s must be %s", name, type ? ((PyTypeObject *)type)->tp_name : "a registered structure");
    }
}

// The bytes behind a ctypes structure or array (a prom_requant, a layer table, a job table).
class Buffer {
public:
    Buffer(PyObject *o, size_t at_least, PyObject *type, const char *name)
    {
        structure(o, type, name);
        if (PyObject_GetBuffer(o, &view_, PyBUF_SIMPLE) != 0) throw ArgError();
        if ((size_t)view_.len < at_least) {
            PyBuffer_Release(&view_);
            PyErr_SetString(PyExc_ValueError, "structure argument too small");
            throw ArgError();
        }
    }
    ~Buffer() { PyBuffer_Release(&view_); }
    Buffer(const Buffer &) = delete;
    Buffer &operator=(const Buffer &) = delete;
    template <class T> const T *as() const { return static_cast<const T *>(view_.buf); }

private:
    Py_buffer view_;
};

// Runs a library call with the interpreter lock released.
template <class F> PyObject *call(F f)
{
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = (int)f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

template <class F> PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        return nullptr;
    }
    try {
        return f();
    } catch (const ArgError &) {
        return nullptr;
    } catch (const std::exception &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// (x, w_packed, cout, rq, y, variant, stream)
PyObject *pw_conv_i8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const at::Tensor &x = dev(a[0], at::kChar, "x");
        dims(x, 2, "x");
        const int64_t m = x.size(0);
        const int cin = (int)x.size(1), cout = small_int(a[2]), variant = small_int(a[5]);
        const auto *xp = ptr<const int8_t>(x);
        const auto *wp = ptr<const uint8_t>(dev(a[1], at::kByte, "w_packed"));
        auto *yp = ptr<int8_t>(dev(a[4], at::kChar, "y"));
        const Buffer rq(a[3], sizeof(prom_requant), requant_type, "rq");
        void *st = stream(a[6]);
        return call([&] { return prom_pw_conv_i8(xp, m, cin, wp, cout, rq.as<prom_requant>(), yp, (prom_variant)variant, st); });
    });
}

// (x, w_packed, cout, rq, res, y, variant, stream)
PyObject *pw_conv_i8_res(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        const at::Tensor &x = dev(a[0], at::kChar, "x");
        dims(x, 2, "x");
        const int64_t m = x.size(0);
        const int cin = (int)x.size(1), cout = small_int(a[2]), variant = small_int(a[6]);
        const at::Tensor &res = dev(a[4], at::kChar, "res");
        if (res.dim() != 2 || res.size(0) != m || res.size(1) != cout) fail(PyExc_ValueError, "%s must be [m, cout]", "res");
        const auto *xp = ptr<const int8_t>(x);
        const auto *wp = ptr<const uint8_t>(dev(a[1], at::kByte, "w_packed"));
        const auto *rp = ptr<const int8_t>(res);
        auto *yp = ptr<int8_t>(dev(a[5], at::kChar, "y"));
        const Buffer rq(a[3], sizeof(prom_requant), requant_type, "rq");
        void *st = stream(a[7]);
        return call([&] { return prom_pw_conv_i8_res(xp, m, cin, wp, cout, rq.as<prom_requant>(), rp, yp, (prom_variant)variant, st); });
    });
}

// (x, cout, prepared, act_min, act_max, y, stream)
PyObject *pw_conv_i8_prepared(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const at::Tensor &x = dev(a[0], at::kChar, "x");
        dims(x, 2, "x");
        const int64_t m = x.size(0);
        const int cin = (int)x.size(1), cout = small_int(a[1]), lo = small_int(a[3]), hi = small_int(a[4]);
        const auto *xp = ptr<const int8_t>(x);
        const void *pp = ptr<const uint8_t>(dev(a[2], at::kByte, "prepared"));
        auto *yp = ptr<int8_t>(dev(a[5], at::kChar, "y"));
        void *st = stream(a[6]);
        return call([&] { return prom_pw_conv_i8_prepared(xp, m, cin, cout, pp, lo, hi, yp, st); });
    });
}

// (x, batch, w_packed, cout, alpha, gamma_x, q, gamma_y, scale_y, stream)
PyObject *pw_conv_i8_dyn(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, [&] {
        const at::Tensor &x = dev(a[0], at::kChar, "x");
        dims(x, 2, "x");
        const int64_t m = x.size(0);
        const int cin = (int)x.size(1), batch = small_int(a[1]), cout = small_int(a[3]);
        if (batch && m % batch) fail(PyExc_ValueError, "%s", "rows must divide evenly into samples");
        const int64_t rows = batch ? m / batch : 1;
        const auto *xp = ptr<const int8_t>(x);
        const auto *wp = ptr<const uint8_t>(dev(a[2], at::kByte, "w_packed"));
        const auto *al = ptr<const float>(dev(a[4], at::kFloat, "alpha"));
        const auto *gx = ptr<const float>(dev(a[5], at::kFloat, "gamma_x"));
        auto *q = ptr<int8_t>(tensor(a[6], "q"));
        auto *gy = ptr<float>(tensor(a[7], "gamma_y"));
        auto *sy = ptr<float>(tensor(a[8], "scale_y"));
        void *st = stream(a[9]);
        return call([&] { return prom_pw_conv_i8_dyn(xp, batch, rows, cin, wp, cout, al, gx, q, gy, sy, st); });
    });
}

// (x, w, rq, stride, y, stream); x is [batch, h, w, c]
PyObject *dw_conv3x3_i8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const at::Tensor &x = dev(a[0], at::kChar, "x");
        dims(x, 4, "x");
        const int b = (int)x.size(0), h = (int)x.size(1), w = (int)x.size(2), c = (int)x.size(3);
        const int stride = small_int(a[3]);
        const auto *xp = ptr<const int8_t>(x);
        const auto *wp = ptr<const int8_t>(dev(a[1], at::kChar, "w"));
        auto *yp = ptr<int8_t>(dev(a[4], at::kChar, "y"));
        const Buffer rq(a[2], sizeof(prom_requant), requant_type, "rq");
        void *st = stream(a[5]);
        return call([&] { return prom_dw_conv3x3_i8(xp, b, h, w, c, stride, wp, rq.as<prom_requant>(), yp, st); });
    });
}

// (x, q, gamma, scale, stream); x is [batch, ...]
PyObject *quantize_act_absmax(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 5, [&] {
        const at::Tensor &x = tensor(a[0], "x"), &q = tensor(a[1], "q"), &g = tensor(a[2], "gamma"), &s = tensor(a[3], "scale");
        if (!x.is_cuda() || x.scalar_type() != at::kFloat || !x.is_contiguous() || x.dim() < 1)
            fail(PyExc_ValueError, "%s must be a contiguous float32 CUDA tensor", "x");
        const int64_t batch = x.size(0);
        if (q.sizes() != x.sizes() || q.scalar_type() != at::kChar || !q.is_cuda() || g.numel() != batch ||
            s.numel() != batch || g.scalar_type() != at::kFloat || s.scalar_type() != at::kFloat)
            fail(PyExc_ValueError, "%s must be (int8 like x, float32 [batch], float32 [batch]) on the device", "out");
        const int64_t per = batch ? x.numel() / batch : 1;
        const auto *xp = ptr<const float>(x);
        auto *qp = ptr<int8_t>(q);
        auto *gp = ptr<float>(g), *sp = ptr<float>(s);
        void *st = stream(a[4]);
        return call([&] { return prom_quantize_act_absmax(xp, (int)batch, per, qp, gp, sp, st); });
    });
}

// (job table, n, stream)
PyObject *quantize_ternary_batch(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 3, [&] {
        const int jobs = small_int(a[1]);
        const Buffer t(a[0], (size_t)(jobs > 0 ? jobs : 0) * sizeof(prom_quantize_job), job_type, "jobs");
        void *st = stream(a[2]);
        return call([&] { return prom_quantize_ternary_batch(t.as<prom_quantize_job>(), jobs, st); });
    });
}

// (layer table, n, x0, workspace, y, variant, stream); x0 is [batch, h, w, cin]
PyObject *pw_layer_seq(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const int layers = small_int(a[1]), variant = small_int(a[5]);
        const at::Tensor &x = dev(a[2], at::kChar, "x0");
        dims(x, 4, "x0");
        const int b = (int)x.size(0), h = (int)x.size(1), w = (int)x.size(2);
        const at::Tensor &ws = tensor(a[3], "workspace");
        const Buffer t(a[0], (size_t)(layers > 0 ? layers : 0) * sizeof(prom_layer), layer_type, "layers");
        const auto *xp = ptr<const int8_t>(x);
        void *wsp = ws.data_ptr();
        const size_t ws_bytes = (size_t)ws.numel();
        auto *yp = ptr<int8_t>(dev(a[4], at::kChar, "y_out"));
        void *st = stream(a[6]);
        return call([&] { return prom_pw_layer_seq(t.as<prom_layer>(), layers, xp, b, h, w, wsp, ws_bytes, yp, (prom_variant)variant, st); });
    });
}

// ---- float matrices: their type, their rows and how far these are apart --------------------------------------
prom_type float_type(const at::Tensor &t, const char *name)
{
    switch (t.scalar_type()) {
    case at::kFloat: return PROM_TYPE_F32;
    case at::kBFloat16: return PROM_TYPE_BF16;
    case at::kHalf: return PROM_TYPE_F16;
    default: fail(PyExc_ValueError, "%s must be float32, bfloat16 or float16", name);
    }
}

// The library launches on the current device: a tensor elsewhere would be another device's pointer there.
void here(const at::Tensor &t, const char *name)
{
    if (!t.is_cuda()) fail(PyExc_ValueError, "%s must be a CUDA tensor", name);
    if (t.device().index() != c10::cuda::current_device()) fail(PyExc_ValueError, "%s must be on the current CUDA device", name);
}

struct Rows {
    void *p;
    prom_type type;
    int64_t m, pitch;
    int n;
};

// [..., n] with dense rows: any pitch between the rows of a matrix, none between those of more dimensions.
Rows rows(PyObject *o, const char *name)
{
    const at::Tensor &t = tensor(o, name);
    here(t, name);
    if (t.dim() < 1) fail(PyExc_ValueError, "%s must have a dimension at least", name);
    const int64_t n = t.size(-1);
    if (n > INT32_MAX) fail(PyExc_ValueError, "%s has too many columns", name);
    if (t.dim() == 2 ? n > 1 && t.stride(1) != 1 : !t.is_contiguous()) fail(PyExc_ValueError, "%s must have dense rows", name);
    int64_t m = 1;
    for (int64_t i = 0; i + 1 < t.dim(); ++i) m *= t.size(i);
    return {t.data_ptr(), float_type(t, name), m, t.dim() == 2 && m > 1 ? t.stride(0) : n, (int)n};
}

void same(const Rows &a, const Rows &b, const char *name)
{
    if (a.m != b.m || a.n != b.n || a.type != b.type) fail(PyExc_ValueError, "%s must have x's shape and type", name);
}

// A dense vector of `n` values of type `t`; None gives no pointer.
void *vector(PyObject *o, int64_t n, at::ScalarType t, const char *name)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &v = dev(o, t, name);
    here(v, name);
    if (v.numel() != n) fail(PyExc_ValueError, "%s has another number of values than the rows need", name);
    return v.data_ptr();
}

// The parameters of a norm have one type: the first one's that is there.
at::ScalarType param_type(PyObject *a, PyObject *b, PyObject *c, prom_type &type)
{
    for (PyObject *o : {a, b, c})
        if (o != Py_None) {
            const at::Tensor &t = tensor(o, "a parameter");
            type = float_type(t, "a parameter");
            return t.scalar_type();
        }
    type = PROM_TYPE_F32;
    return at::kFloat;
}

double real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw ArgError();
    return v;
}

// (x, weight, bias, eps, y, mean, rstd, stream)
PyObject *layer_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        const Rows x = rows(a[0], "x"), y = rows(a[4], "y");
        same(x, y, "y");
        prom_type pt;
        const at::ScalarType pts = param_type(a[1], a[2], Py_None, pt);
        const void *w = vector(a[1], x.n, pts, "weight"), *b = vector(a[2], x.n, pts, "bias");
        const double eps = real(a[3]);
        auto *mean = static_cast<float *>(vector(a[5], x.m, at::kFloat, "mean"));
        auto *rstd = static_cast<float *>(vector(a[6], x.m, at::kFloat, "rstd"));
        void *st = stream(a[7]);
        return call([&] { return prom_layer_norm(x.p, x.type, x.m, x.n, x.pitch, w, b, pt, eps, y.p, y.pitch, mean, rstd, st); });
    });
}

// (x, weight, bias, eps, q, gamma, scale, mean, rstd, stream)
PyObject *layer_norm_i8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, [&] {
        const Rows x = rows(a[0], "x");
        prom_type pt;
        const at::ScalarType pts = param_type(a[1], a[2], Py_None, pt);
        const void *w = vector(a[1], x.n, pts, "weight"), *b = vector(a[2], x.n, pts, "bias");
        const double eps = real(a[3]);
        auto *q = static_cast<int8_t *>(vector(a[4], x.m * x.n, at::kChar, "q"));
        auto *gamma = static_cast<float *>(vector(a[5], x.m, at::kFloat, "gamma"));
        auto *scale = static_cast<float *>(vector(a[6], x.m, at::kFloat, "scale"));
        auto *mean = static_cast<float *>(vector(a[7], x.m, at::kFloat, "mean"));
        auto *rstd = static_cast<float *>(vector(a[8], x.m, at::kFloat, "rstd"));
        void *st = stream(a[9]);
        return call([&] { return prom_layer_norm_i8(x.p, x.type, x.m, x.n, x.pitch, w, b, pt, eps, q, gamma, scale, mean, rstd, st); });
    });
}

// A call's workspace: the caller's tensor, or memory of PyTorch's pool that belongs to the stream the call runs on and goes
// back to it when the call has been enqueued (what the stream is given next runs behind the call).
class Workspace {
public:
    Workspace(PyObject *given, size_t bytes, void *st)
    {
        if (given != Py_None) {
            const at::Tensor &t = dev(given, at::kByte, "workspace");
            here(t, "workspace");
            p = t.data_ptr();
            size = (size_t)t.numel();
        } else if (bytes) {
            try {
                p = own_ = c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(bytes, static_cast<cudaStream_t>(st));
            } catch (const std::exception &e) {
                PyErr_SetString(PyExc_MemoryError, e.what());
                throw ArgError();
            }
            size = bytes;
        }
    }
    ~Workspace() { if (own_) c10::cuda::CUDACachingAllocator::raw_delete(own_); }
    Workspace(const Workspace &) = delete;
    Workspace &operator=(const Workspace &) = delete;
    void *p = nullptr;
    size_t size = 0;

private:
    void *own_ = nullptr;
};

// (dy, x, weight, mean, rstd, dx, dweight, dbias, workspace, stream)
PyObject *layer_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, [&] {
        const Rows x = rows(a[1], "x"), dy = rows(a[0], "dy");
        same(x, dy, "dy");
        Rows dx{nullptr, x.type, x.m, x.n, x.n};
        if (a[5] != Py_None) {
            dx = rows(a[5], "dx");
            same(x, dx, "dx");
        }
        prom_type pt;
        const at::ScalarType pts = param_type(a[2], a[6], a[7], pt);
        const void *w = vector(a[2], x.n, pts, "weight");
        const auto *mean = static_cast<const float *>(vector(a[3], x.m, at::kFloat, "mean"));
        const auto *rstd = static_cast<const float *>(vector(a[4], x.m, at::kFloat, "rstd"));
        void *dw = vector(a[6], x.n, pts, "dweight"), *db = vector(a[7], x.n, pts, "dbias");
        void *st = stream(a[9]);
        const Workspace ws(a[8], dw || db ? prom_layer_norm_backward_workspace_bytes(x.m, x.n) : 0, st);
        return call([&] {
            return prom_layer_norm_backward(dy.p, x.p, x.type, x.m, x.n, dy.pitch, x.pitch, w, pt, mean, rstd, dx.p, dx.pitch,
                                            dw, db, ws.p, ws.size, st);
        });
    });
}

// (x, batch, w_packed, cout, alpha, gamma_x, a, b, scale, adapter_of_sample, y, workspace, stream); a None: no adapters
PyObject *pw_proj_adapters(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 13, [&] {
        const at::Tensor &x = dev(a[0], at::kChar, "x"), &w = dev(a[2], at::kByte, "w_packed");
        dims(x, 2, "x");
        here(x, "x");
        here(w, "w_packed");
        const int batch = small_int(a[1]), cout = small_int(a[3]);
        const int64_t m = x.size(0), cin = x.size(1);
        if (batch < 0 || (batch ? m % batch != 0 || m == 0 : m != 0)) fail(PyExc_ValueError, "%s must have a whole number of rows per sample", "x");
        if (cin > INT32_MAX || cout < 0 || w.numel() != cout * ((cin + 3) / 4))
            fail(PyExc_ValueError, "%s must have cout rows of ceil(cin / 4) bytes", "w_packed");
        const auto *alpha = static_cast<const float *>(vector(a[4], cout, at::kFloat, "alpha"));
        const auto *gamma = static_cast<const float *>(vector(a[5], batch, at::kFloat, "gamma_x"));
        prom_adapters ad{nullptr, nullptr, nullptr, PROM_TYPE_BF16, 0, 1};
        const int32_t *which = nullptr;
        if (a[6] != Py_None) {
            const at::Tensor &av = tensor(a[6], "a"), &bv = tensor(a[7], "b");
            ad.type = float_type(av, "a");
            if (ad.type == PROM_TYPE_F32) fail(PyExc_ValueError, "%s must be bfloat16 or float16", "a");
            dev(a[6], av.scalar_type(), "a");
            dev(a[7], av.scalar_type(), "b");
            here(av, "a");
            here(bv, "b");
            dims(av, 3, "a");
            dims(bv, 3, "b");
            if (av.size(2) != cin) fail(PyExc_ValueError, "%s must be [adapters, rank, cin]", "a");
            if (bv.size(0) != av.size(0) || bv.size(1) != cout || bv.size(2) != av.size(1))
                fail(PyExc_ValueError, "%s must be [adapters, cout, rank]", "b");
            if (av.size(0) > INT32_MAX || av.size(1) > INT32_MAX) fail(PyExc_ValueError, "%s has too many rows", "a");
            ad.n = (int)av.size(0);
            ad.rank = (int)av.size(1);
            ad.a_dev = av.data_ptr();
            ad.b_dev = bv.data_ptr();
            ad.scale_dev = static_cast<const float *>(vector(a[8], ad.n, at::kFloat, "scale"));
            which = static_cast<const int32_t *>(vector(a[9], batch, at::kInt, "adapter_of_sample"));
        }
        const Rows y = rows(a[10], "y");
        if (y.m != m || y.n != cout) fail(PyExc_ValueError, "%s must be [rows of x, cout]", "y");
        void *st = stream(a[12]);
        const Workspace ws(a[11], ad.n ? prom_pw_proj_adapters_workspace_bytes(batch, batch ? m / batch : 1, ad.rank) : 0, st);
        const auto *xp = ptr<const int8_t>(x);
        const auto *wp = ptr<const uint8_t>(w);
        return call([&] {
            return prom_pw_proj_adapters(xp, batch, batch ? m / batch : 1, (int)cin, wp, cout, alpha, gamma, &ad, which, y.p,
                                         y.type, y.pitch, ws.p, ws.size, st);
        });
    });
}

// (prom_requant, prom_layer, prom_quantize_job as the binding has them); kept for as long as the module
PyObject *register_types(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 3, [&] {
        for (int i = 0; i < 3; ++i) {
            if (!PyType_Check(a[i])) fail(PyExc_TypeError, "%s", "types are expected");
            Py_INCREF(a[i]);
        }
        requant_type = a[0]; layer_type = a[1]; job_type = a[2];
        Py_RETURN_NONE;
    });
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(pw_conv_i8), ENTRY(pw_conv_i8_res), ENTRY(pw_conv_i8_prepared), ENTRY(pw_conv_i8_dyn),
                         ENTRY(dw_conv3x3_i8), ENTRY(quantize_act_absmax), ENTRY(quantize_ternary_batch),
                         ENTRY(pw_layer_seq), ENTRY(layer_norm), ENTRY(layer_norm_i8), ENTRY(layer_norm_backward),
                         ENTRY(pw_proj_adapters),
                         ENTRY(register_types), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
