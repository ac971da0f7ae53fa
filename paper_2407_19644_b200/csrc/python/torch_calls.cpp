// Argument checks and output allocation of the token-major calls (ubp_rmsnorm, ubp_quant_rows, ubp_linear,
// ubp_rotate_append, ubp_attention), compiled against
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

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "ubp.h"

namespace {

decltype(&ubp_rmsnorm) p_rmsnorm = nullptr;
decltype(&ubp_quant_rows) p_quant_rows = nullptr;
decltype(&ubp_linear) p_linear = nullptr;
decltype(&ubp_linear_workspace_size) p_workspace = nullptr;
decltype(&ubp_rotate_append) p_rotate_append = nullptr;
decltype(&ubp_attention) p_attention = nullptr;
decltype(&ubp_attention_workspace_size) p_attention_workspace = nullptr;

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
        count(n, 7);
        void *p[7];
        for (int i = 0; i < 7; ++i) if (!(p[i] = PyLong_AsVoidPtr(a[i]))) throw Refused();
        p_rmsnorm = reinterpret_cast<decltype(p_rmsnorm)>(p[0]);
        p_quant_rows = reinterpret_cast<decltype(p_quant_rows)>(p[1]);
        p_linear = reinterpret_cast<decltype(p_linear)>(p[2]);
        p_workspace = reinterpret_cast<decltype(p_workspace)>(p[3]);
        p_rotate_append = reinterpret_cast<decltype(p_rotate_append)>(p[4]);
        p_attention = reinterpret_cast<decltype(p_attention)>(p[5]);
        p_attention_workspace = reinterpret_cast<decltype(p_attention_workspace)>(p[6]);
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

// k_cache, v_cache, page_table, lengths and starts as the library's description of a cache; T rows are given.
ubp_cache_t cache_of(const at::Tensor *k, const at::Tensor *v, const at::Tensor *table, const at::Tensor *lengths, const at::Tensor *starts, int64_t T)
{
    if (!k || !k->is_cuda() || k->dim() != 4 || (k->scalar_type() != at::kBFloat16 && k->scalar_type() != at::kHalf))
        refuse("k_cache must be a [pages][heads][page size][head size] bfloat16 or float16 CUDA tensor");
    const int dev = k->get_device();
    if (!v || !v->is_cuda() || v->get_device() != dev || v->scalar_type() != k->scalar_type() || v->sizes() != k->sizes() || v->strides() != k->strides())
        refuse("v_cache must have k_cache's type, device, sizes and strides");
    for (int i = 0; i < 4; ++i) if (k->size(i) < 1 || k->size(i) > INT32_MAX) refuse("k_cache must have pages, heads, tokens and values");
    if (k->stride(3) != 1 && k->size(3) > 1) refuse("the values of a token in the cache must be contiguous");
    if (!table || !table->is_cuda() || table->get_device() != dev || table->scalar_type() != at::kInt || table->dim() != 2 ||
        (table->size(1) > 1 && table->stride(1) != 1) || table->size(1) < 1 || table->size(1) > INT32_MAX)
        refuse("page_table must be a [sequences][pages of a sequence] int32 tensor with contiguous rows on cuda:" + std::to_string(dev));
    const int64_t B = table->size(0);
    if (!lengths) refuse("lengths is required");
    ubp_cache_t c{};
    c.k = k->data_ptr(); c.v = v->data_ptr();
    c.page_stride = k->stride(0); c.head_stride = k->stride(1); c.token_stride = k->stride(2);
    c.pages = k->size(0); c.kv_heads = (int)k->size(1); c.page_size = (int)k->size(2); c.head_dim = (int)k->size(3);
    c.dtype = code_of(k->scalar_type());
    c.table = table->data_ptr<int32_t>(); c.table_stride = table->stride(0); c.table_width = (int)table->size(1);
    c.batch = B;
    c.lengths = static_cast<const int32_t *>(vec(*lengths, "lengths", B, at::kInt, dev));
    if (starts) c.starts = static_cast<const int32_t *>(vec(*starts, "starts", B + 1, at::kInt, dev));
    else if (T != B) refuse("without starts there is one new token a sequence");
    // (a stride that is never used may be anything in a tensor, and has to be a possible one here)
    if (c.page_size == 1) c.token_stride = c.head_dim;
    if (c.pages == 1) c.page_stride = 0;
    if (c.kv_heads == 1) c.head_stride = 0;
    return c;
}
// a [T][H][D] tensor of the cache's type and device; strides between tokens and heads
void heads(const at::Tensor &t, const char *name, int64_t T, int64_t H, int64_t D, at::ScalarType type, int dev, int64_t &ts, int64_t &hs)
{
    if (t.dim() != 3 || t.size(0) != T || t.size(1) != H || t.size(2) != D || t.scalar_type() != type || !t.is_cuda() || t.get_device() != dev)
        refuse(std::string(name) + " must be a [" + std::to_string(T) + "][" + std::to_string(H) + "][" + std::to_string(D) + "] tensor of " +
               c10::toString(type) + " on cuda:" + std::to_string(dev));
    ts = T > 1 ? t.stride(0) : H * D;
    hs = H > 1 ? t.stride(1) : D;
    if ((D > 1 && t.stride(2) != 1) || hs < D || ts < D) refuse(std::string(name) + " must have contiguous heads that do not overlap");
}
at::Tensor make(int64_t T, int64_t H, int64_t D, at::ScalarType type, int dev)
{
    return at::detail::empty_cuda({T, H, D}, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)dev), std::nullopt);
}

// rotate_append(qkv, q_heads, k_cache, v_cache, page_table, lengths, starts, rotation, interleaved, q_gamma, k_gamma, eps, out, stream)
PyObject *rotate_append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        count(n, 14);
        const at::Tensor *qkv = tensor(a[0], "qkv"), *k = tensor(a[2], "k_cache"), *starts = tensor(a[6], "starts"), *rot = tensor(a[7], "rotation"),
                         *qg = tensor(a[9], "q_gamma"), *kg = tensor(a[10], "k_gamma"), *out = tensor(a[12], "out");
        const int64_t Hq = PyLong_AsLongLong(a[1]);
        const int inter = PyObject_IsTrue(a[8]);
        const double eps = PyFloat_AsDouble(a[11]);
        if (PyErr_Occurred()) throw Refused();
        if (!qkv || qkv->dim() != 2) refuse("qkv must be a [T][heads * head size] CUDA tensor");
        const int64_t T = qkv->size(0);
        const ubp_cache_t c = cache_of(k, tensor(a[3], "v_cache"), tensor(a[4], "page_table"), tensor(a[5], "lengths"), starts, T);
        const int dev = k->get_device();
        const at::ScalarType type = k->scalar_type();
        if (Hq < 1 || Hq > INT32_MAX || Hq % c.kv_heads) refuse("q_heads must be a multiple of the cache's heads");
        const int64_t D = c.head_dim, ld = rows(*qkv, "qkv", T, (Hq + 2 * (int64_t)c.kv_heads) * D, type, dev);
        const void *pqg = qg ? vec(*qg, "q_gamma", D, type, dev) : nullptr, *pkg = kg ? vec(*kg, "k_gamma", D, type, dev) : nullptr;
        if (rot && (rot->dim() != 2 || rot->scalar_type() != at::kFloat || !rot->is_cuda() || rot->get_device() != dev || rot->size(0) < 1 || rot->size(1) < 2 ||
                    rot->size(1) > D || rot->size(1) % 2 || rot->stride(1) != 1 || (rot->size(0) > 1 && rot->stride(0) < rot->size(1))))
            refuse("rotation must be a [positions][rotated values] float32 tensor with contiguous rows on cuda:" + std::to_string(dev) +
                   ", an even number of them up to the head size");
        int64_t ts = Hq * D, hs = D;
        if (out) heads(*out, "out", T, Hq, D, type, dev, ts, hs);
        if (out && T > 0 && out->data_ptr() == qkv->data_ptr() && ((T > 1 && ts != ld) || (Hq > 1 && hs != D)))
            refuse("out starts at qkv's place but is not the queries' own place in it");
        On on(dev, a[13]);
        at::Tensor q;
        if (!out) q = make(T, Hq, D, type, dev);
        const int rc = p_rotate_append(&c, qkv->data_ptr(), ld, T, (int)Hq, pqg, pkg, (float)eps, rot ? rot->data_ptr<float>() : nullptr, rot ? rot->stride(0) : 0,
                                       rot ? rot->size(0) : 0, rot ? (int)rot->size(1) : 0, inter, out ? out->data_ptr() : q.data_ptr(), ts, hs, on.stream);
        if (rc) return PyLong_FromLong(rc);
        return give(a[12], std::move(q));
    });
}

// attention(q, k_cache, v_cache, page_table, lengths, starts, prefix, window, sinks, scale, max_new, out, stream, workspace)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        count(n, 14);
        const at::Tensor *q = tensor(a[0], "q"), *k = tensor(a[1], "k_cache"), *starts = tensor(a[5], "starts"), *out = tensor(a[11], "out"),
                         *ws = tensor(a[13], "workspace");
        const int64_t prefix = PyLong_AsLongLong(a[6]), window = PyLong_AsLongLong(a[7]), sinks = PyLong_AsLongLong(a[8]);
        if (PyErr_Occurred()) throw Refused();
        if (!q || q->dim() != 3) refuse("q must be a [T][heads][head size] CUDA tensor");
        const int64_t T = q->size(0), Hq = q->size(1);
        const ubp_cache_t c = cache_of(k, tensor(a[2], "v_cache"), tensor(a[3], "page_table"), tensor(a[4], "lengths"), starts, T);
        const double scale = a[9] == Py_None ? 1.0 / std::sqrt((double)c.head_dim) : PyFloat_AsDouble(a[9]);
        const int64_t most = a[10] == Py_None ? std::max<int64_t>(1, starts ? T : 1) : PyLong_AsLongLong(a[10]);
        if (PyErr_Occurred()) throw Refused();
        const int dev = k->get_device();
        const at::ScalarType type = k->scalar_type();
        if (Hq < 1 || Hq > INT32_MAX || Hq % c.kv_heads) refuse("q's heads must be a multiple of the cache's heads");
        if (window < 0 || window > INT32_MAX || sinks < 0 || sinks > INT32_MAX) refuse("window and sinks must be numbers of tokens");
        int64_t qts, qhs, ots = Hq * c.head_dim, ohs = c.head_dim;
        heads(*q, "q", T, Hq, c.head_dim, type, dev, qts, qhs);
        if (out) heads(*out, "out", T, Hq, c.head_dim, type, dev, ots, ohs);
        if (out && T > 0 && out->data_ptr() == q->data_ptr()) refuse("out must not be q: heads of a group read each other's queries");
        if (ws && (!ws->is_cuda() || ws->get_device() != dev || !ws->is_contiguous())) refuse("workspace must be a contiguous tensor on the cache's device");
        On on(dev, a[12]);
        at::Tensor y, room;
        if (!out) y = make(T, Hq, c.head_dim, type, dev);
        void *pw = ws ? ws->data_ptr() : nullptr;
        size_t nws = ws ? ws->numel() * ws->element_size() : 0;
        if (!ws && (nws = p_attention_workspace(&c, q->data_ptr(), qts, qhs, T, (int)Hq, (int)window, (int)sinks, prefix, most)) != 0) {
            room = make((int64_t)nws, at::kByte, dev);
            pw = room.data_ptr();
        }
        const int rc = p_attention(&c, q->data_ptr(), qts, qhs, T, (int)Hq, (float)scale, (int)window, (int)sinks, prefix, most, out ? out->data_ptr() : y.data_ptr(),
                                   ots, ohs, pw, nws, on.stream);
        if (rc) return PyLong_FromLong(rc);
        return give(a[11], std::move(y));
    });
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "addresses of ubp_rmsnorm, ubp_quant_rows, ubp_linear, ubp_linear_workspace_size, ubp_rotate_append, ubp_attention, "
     "ubp_attention_workspace_size"},
    {"rmsnorm", (PyCFunction)(void (*)(void))rmsnorm, METH_FASTCALL, "rmsnorm(x, gamma, eps, residual, out_dtype, out, scales, residual_out, stream)"},
    {"quant_rows", (PyCFunction)(void (*)(void))quant_rows, METH_FASTCALL, "quant_rows(x, out, scales, stream)"},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL,
     "linear(plan, x, bias, activation, residual, x_scales, out, out_dtype, stream, workspace)"},
    {"rotate_append", (PyCFunction)(void (*)(void))rotate_append, METH_FASTCALL,
     "rotate_append(qkv, q_heads, k_cache, v_cache, page_table, lengths, starts, rotation, interleaved, q_gamma, k_gamma, eps, out, stream)"},
    {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL,
     "attention(q, k_cache, v_cache, page_table, lengths, starts, prefix, window, sinks, scale, max_new, out, stream, workspace)"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() { return PyModule_Create(&module); }
