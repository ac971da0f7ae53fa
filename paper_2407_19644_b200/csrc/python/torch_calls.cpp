// Argument checks and output allocation of the token-major calls (ubp_rmsnorm, ubp_quant_rows, ubp_linear), compiled against
// torch: a call on one token is bound by the host, and marshalling it in Python cost as much again as the launch (a product 8.2 us
// a call through ctypes, 4.0 here; a norm with 8-bit rows 13.3 and 5.2). The library is still reached through its C
// ABI: bind() receives the addresses of its entry points, so that whichever build of it the package loaded is the one that runs.
// A call returns its outputs, or the library's negative status; refusals of arguments raise ValueError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <string>

#include "ubp.h"

namespace {

decltype(&ubp_rmsnorm) p_rmsnorm = nullptr;
decltype(&ubp_quant_rows) p_quant_rows = nullptr;
decltype(&ubp_linear) p_linear = nullptr;
decltype(&ubp_linear_workspace_size) p_workspace = nullptr;

struct Refused {};                      // a Python exception is set

[[noreturn]] void refuse(const std::string &what)
{
    PyErr_SetString(PyExc_ValueError, what.c_str());
    throw Refused();
}

int code_of(at::ScalarType t)
{
    switch (t) {
        case at::kFloat: return UBP_F32;
        case at::kHalf: return UBP_F16;
        case at::kBFloat16: return UBP_BF16;
        case at::kFloat8_e4m3fn: return UBP_E4M3;
        default: return -1;
    }
}
at::ScalarType type_of(int code)
{
    return code == UBP_F32 ? at::kFloat : code == UBP_F16 ? at::kHalf : code == UBP_BF16 ? at::kBFloat16 : at::kFloat8_e4m3fn;
}

const at::Tensor *tensor(PyObject *o, const char *name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a CUDA tensor");
    return &THPVariable_Unpack(o);
}

// a [T][C] matrix of one type on device `dev` whose rows are contiguous and disjoint; returns its row stride
int64_t rows(const at::Tensor &t, const char *name, int64_t T, int64_t C, at::ScalarType type, int dev)
{
    if (t.dim() != 2 || t.size(0) != T || t.size(1) != C || t.scalar_type() != type || !t.is_cuda() || t.get_device() != dev)
        refuse(std::string(name) + " must be a [" + std::to_string(T) + "][" + std::to_string(C) + "] tensor of " + c10::toString(type) +
               " on cuda:" + std::to_string(dev));
    const int64_t ld = t.stride(0);
    if ((C > 1 && t.stride(1) != 1) || (T > 1 && ld < C)) refuse(std::string(name) + " must have contiguous rows that do not overlap");
    return ld;
}
// Two operands in one place: only element by element, so with one row stride.
void same_rows(const at::Tensor *a, int64_t lda, const at::Tensor *b, int64_t ldb, int64_t T, const char *what)
{
    if (a && b && T > 1 && lda != ldb && a->data_ptr() == b->data_ptr()) refuse(std::string(what) + " start at one place but differ in their row stride");
}
// a contiguous [n] vector
void *vec(const at::Tensor &t, const char *name, int64_t n, at::ScalarType type, int dev)
{
    if (t.dim() != 1 || t.size(0) != n || t.scalar_type() != type || !t.is_cuda() || t.get_device() != dev || (n > 1 && t.stride(0) != 1))
        refuse(std::string(name) + " must be a contiguous [" + std::to_string(n) + "] vector of " + c10::toString(type) + " on cuda:" + std::to_string(dev));
    return t.data_ptr();
}

struct X { int64_t T, C, ld; int dev, code; at::ScalarType type; };
X activations(const at::Tensor *x)
{
    X r;
    r.code = x && x->is_cuda() && x->dim() == 2 ? code_of(x->scalar_type()) : -1;
    if (r.code < 0 || r.code == UBP_E4M3) refuse("x must be a [T][C] float32, float16 or bfloat16 CUDA tensor");
    r.T = x->size(0); r.C = x->size(1); r.dev = x->get_device(); r.type = x->scalar_type();
    r.ld = rows(*x, "x", r.T, r.C, r.type, r.dev);
    if (r.C > INT32_MAX) refuse("x has too many columns");
    return r;
}

// The stream a call runs on: the caller's handle, or the device's current stream. A given stream is the current one while the
// call allocates: memory that the allocator has handed back from another stream may still be in use there.
struct On {
    c10::cuda::OptionalCUDAGuard guard;
    c10::cuda::OptionalCUDAStreamGuard current;
    void *stream;
    On(int dev, PyObject *given) : guard(c10::Device(c10::kCUDA, (c10::DeviceIndex)dev))
    {
        const auto d = (c10::DeviceIndex)dev;
        if (given != Py_None) {
            stream = PyLong_AsVoidPtr(given);
            if (!stream && PyErr_Occurred()) throw Refused();
            current.reset_stream(stream ? c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), d) : c10::cuda::getDefaultCUDAStream(d));
        } else {
            stream = c10::cuda::getCurrentCUDAStream(d).stream();
        }
    }
};

at::Tensor make(int64_t T, int64_t C, at::ScalarType type, int dev)
{
    return at::detail::empty_cuda({T, C}, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)dev), std::nullopt);
}
at::Tensor make(int64_t T, at::ScalarType type, int dev)
{
    return at::detail::empty_cuda({T}, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)dev), std::nullopt);
}

// the given output, or a new tensor
PyObject *give(PyObject *given, at::Tensor &&made)
{
    if (given != Py_None) { Py_INCREF(given); return given; }
    return THPVariable_Wrap(std::move(made));
}

at::ScalarType dtype(PyObject *o, at::ScalarType otherwise)
{
    if (o == Py_None) return otherwise;
    if (!THPDtype_Check(o)) refuse("out_dtype must be a torch dtype");
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

void count(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); throw Refused(); }
}

template <typename Fn> PyObject *guarded(Fn &&fn)
{
    try { return fn(); }
    catch (const Refused &) { return nullptr; }
    catch (const c10::Error &e) { PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace()); return nullptr; }
    catch (const std::exception &e) { PyErr_SetString(PyExc_RuntimeError, e.what()); return nullptr; }
}

PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        count(n, 4);
        void *p[4];
        for (int i = 0; i < 4; ++i) if (!(p[i] = PyLong_AsVoidPtr(a[i]))) throw Refused();
        p_rmsnorm = reinterpret_cast<decltype(p_rmsnorm)>(p[0]);
        p_quant_rows = reinterpret_cast<decltype(p_quant_rows)>(p[1]);
        p_linear = reinterpret_cast<decltype(p_linear)>(p[2]);
        p_workspace = reinterpret_cast<decltype(p_workspace)>(p[3]);
        Py_RETURN_NONE;
    });
}

// rmsnorm(x, gamma, eps, residual, out_dtype, out, scales, residual_out, stream)
PyObject *rmsnorm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        count(n, 9);
        const X x = activations(tensor(a[0], "x"));
        const at::Tensor *gamma = tensor(a[1], "gamma"), *residual = tensor(a[3], "residual"), *out = tensor(a[5], "out"),
                         *scales = tensor(a[6], "scales"), *rout = tensor(a[7], "residual_out");
        const double eps = PyFloat_AsDouble(a[2]);
        if (eps == -1.0 && PyErr_Occurred()) throw Refused();
        if (!gamma) refuse("gamma is required");
        const at::ScalarType gtype = gamma->scalar_type() == at::kFloat ? at::kFloat : x.type;
        const void *pg = vec(*gamma, "gamma", x.C, gtype, x.dev);
        const at::ScalarType type = dtype(a[4], out ? out->scalar_type() : x.type);
        const bool q = type == at::kFloat8_e4m3fn;
        if (!q && type != x.type) refuse("out_dtype must be x's type or torch.float8_e4m3fn");
        const int64_t ldy = out ? rows(*out, "out", x.T, x.C, type, x.dev) : x.C;
        const int64_t ldr = residual ? rows(*residual, "residual", x.T, x.C, x.type, x.dev) : 0;
        int64_t ldh = rout ? rows(*rout, "residual_out", x.T, x.C, x.type, x.dev) : x.C;
        void *ps = q && scales ? vec(*scales, "scales", x.T, at::kFloat, x.dev) : nullptr;
        same_rows(rout, ldh, tensor(a[0], "x"), x.ld, x.T, "residual_out and x");
        same_rows(rout, ldh, residual, ldr, x.T, "residual_out and residual");
        if (out && rout && x.T > 0 && out->data_ptr() == rout->data_ptr()) refuse("out and residual_out are one place");
        On on(x.dev, a[8]);
        at::Tensor y, s, h;
        if (!out) y = make(x.T, x.C, type, x.dev);
        if (q && !scales) { s = make(x.T, at::kFloat, x.dev); ps = s.data_ptr(); }
        if (residual && !rout) h = make(x.T, x.C, x.type, x.dev);
        void *ph = rout ? rout->data_ptr() : residual ? h.data_ptr() : nullptr;
        const int rc = p_rmsnorm(THPVariable_Unpack(a[0]).data_ptr(), x.ld, residual ? residual->data_ptr() : nullptr, ldr, pg, code_of(gtype), x.code,
                                 x.T, (int)x.C, (float)eps, ph, ldh, out ? out->data_ptr() : y.data_ptr(), ldy, code_of(type), (float *)ps, on.stream);
        if (rc) return PyLong_FromLong(rc);
        PyObject *t = PyTuple_New(3);
        if (!t) return nullptr;
        PyTuple_SET_ITEM(t, 0, give(a[5], std::move(y)));
        if (q) PyTuple_SET_ITEM(t, 1, give(a[6], std::move(s)));
        else { Py_INCREF(Py_None); PyTuple_SET_ITEM(t, 1, Py_None); }
        if (ph || rout) PyTuple_SET_ITEM(t, 2, give(a[7], std::move(h)));
        else if (residual) PyTuple_SET_ITEM(t, 2, give(a[7], std::move(h)));       // (no rows: no address)
        else { Py_INCREF(Py_None); PyTuple_SET_ITEM(t, 2, Py_None); }
        return t;
    });
}

// quant_rows(x, out, scales, stream)
PyObject *quant_rows(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        count(n, 4);
        const X x = activations(tensor(a[0], "x"));
        const at::Tensor *out = tensor(a[1], "out"), *scales = tensor(a[2], "scales");
        const int64_t ldq = out ? rows(*out, "out", x.T, x.C, at::kFloat8_e4m3fn, x.dev) : x.C;
        void *ps = scales ? vec(*scales, "scales", x.T, at::kFloat, x.dev) : nullptr;
        On on(x.dev, a[3]);
        at::Tensor q, s;
        if (!out) q = make(x.T, x.C, at::kFloat8_e4m3fn, x.dev);
        if (!scales) { s = make(x.T, at::kFloat, x.dev); ps = s.data_ptr(); }
        const int rc = p_quant_rows(THPVariable_Unpack(a[0]).data_ptr(), x.ld, x.code, x.T, (int)x.C, out ? out->data_ptr() : q.data_ptr(), ldq, (float *)ps, on.stream);
        if (rc) return PyLong_FromLong(rc);
        PyObject *t = PyTuple_New(2);
        if (!t) return nullptr;
        PyTuple_SET_ITEM(t, 0, give(a[1], std::move(q)));
        PyTuple_SET_ITEM(t, 1, give(a[2], std::move(s)));
        return t;
    });
}

// linear((handle, M, C, F, type code, device, the buffer's stream, the buffer), x, bias, activation code, residual, x_scales, out, out_dtype, stream, workspace)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        count(n, 10);
        if (!PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != 8) { PyErr_SetString(PyExc_TypeError, "bad plan"); throw Refused(); }
        const auto *plan = static_cast<const ubp_linear_plan_t *>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], 0)));
        int64_t d[5];
        for (int i = 0; i < 5; ++i) d[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(a[0], i + 1));
        void *home = PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], 6));
        const long act = PyLong_AsLong(a[3]);
        if (PyErr_Occurred()) throw Refused();
        const int64_t M = d[0], C = d[1], F = d[2];
        const int code = (int)d[3], dev = (int)d[4];
        const bool q = code == UBP_E4M3;
        const at::Tensor *x = tensor(a[1], "x"), *bias = tensor(a[2], "bias"), *residual = tensor(a[4], "residual"), *xs = tensor(a[5], "x_scales"),
                         *out = tensor(a[6], "out"), *ws = tensor(a[9], "workspace");
        if (!x || x->dim() != 2) refuse("x must be a [T][C] CUDA tensor");
        const int64_t T = x->size(0), ldx = rows(*x, "x", T, C, type_of(code), dev);
        if (q != (xs != nullptr)) refuse("x_scales goes with an 8-bit plan");
        const void *ps = xs ? vec(*xs, "x_scales", T, at::kFloat, dev) : nullptr, *pb = bias ? vec(*bias, "bias", M, at::kFloat, dev) : nullptr;
        const at::ScalarType type = dtype(a[7], out ? out->scalar_type() : q ? at::kBFloat16 : type_of(code));
        const int ydt = code_of(type);
        if (ydt < 0) refuse("out_dtype must be float32, float16 or bfloat16");
        const int64_t ldy = out ? rows(*out, "out", T, F, type, dev) : F, ldr = residual ? rows(*residual, "residual", T, F, type, dev) : 0;
        if (out && T > 0 && out->data_ptr() == x->data_ptr()) refuse("out must not be x: every output reads a whole row of it");
        same_rows(out, ldy, residual, ldr, T, "out and residual");
        if (ws && (!ws->is_cuda() || ws->get_device() != dev || !ws->is_contiguous())) refuse("workspace must be a contiguous tensor on the plan's device");
        On on(dev, a[8]);
        if (on.stream != home)              // the plan's memory is in use on this stream too
            c10::cuda::CUDACachingAllocator::recordStream(tensor(PyTuple_GET_ITEM(a[0], 7), "the plan's buffer")->storage().data_ptr(),
                                                          c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev));
        at::Tensor y, room;
        if (!out) y = make(T, F, type, dev);
        const void *px = x->data_ptr();
        void *pw = ws ? ws->data_ptr() : nullptr;
        size_t nws = ws ? ws->numel() * ws->element_size() : 0;
        if (!ws && (nws = p_workspace(plan, px, ldx, T)) != 0) {
            room = make((int64_t)nws, at::kByte, dev);
            pw = room.data_ptr();
        }
        const int rc = p_linear(plan, px, ldx, (const float *)ps, T, (const float *)pb, (int)act, residual ? residual->data_ptr() : nullptr, ldr,
                                out ? out->data_ptr() : y.data_ptr(), ldy, ydt, pw, nws, on.stream);
        if (rc) return PyLong_FromLong(rc);
        return give(a[6], std::move(y));
    });
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "addresses of ubp_rmsnorm, ubp_quant_rows, ubp_linear, ubp_linear_workspace_size"},
    {"rmsnorm", (PyCFunction)(void (*)(void))rmsnorm, METH_FASTCALL, "rmsnorm(x, gamma, eps, residual, out_dtype, out, scales, residual_out, stream)"},
    {"quant_rows", (PyCFunction)(void (*)(void))quant_rows, METH_FASTCALL, "quant_rows(x, out, scales, stream)"},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL,
     "linear(plan, x, bias, activation, residual, x_scales, out, out_dtype, stream, workspace)"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() { return PyModule_Create(&module); }
