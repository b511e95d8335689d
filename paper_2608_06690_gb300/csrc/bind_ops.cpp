// The operators around the layer as Python functions over PyTorch's tensors:
// checks of the arguments, outputs and scratch from the caching allocator, and
// the call of the C ABI (include/pmpe.h) on the current stream of the tensors'
// device.  pmpe.py holds the public functions, their defaults and documents.
//
// Why C++: at decode sizes a call is its host time (1.75 us of kernel for one
// token's norm).  Checks, three allocations and the launch took 8 us in a loop
// of calls from Python through ctypes on a Grace core, 4.4 us from here;
// clipping four tensors 19.8 and 7.9 us.
#include <Python.h>

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <cstring>
#include <initializer_list>
#include <utility>
#include <vector>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "pmpe.h"

namespace {

// The library's functions (pmpe.py passes the addresses of those it loaded).
decltype(&pmpe_rms_norm) lib_rms_norm;
decltype(&pmpe_rms_norm_backward_workspace_size) lib_rms_norm_backward_workspace_size;
decltype(&pmpe_rms_norm_backward) lib_rms_norm_backward;
decltype(&pmpe_route) lib_route;
decltype(&pmpe_route_backward) lib_route_backward;
decltype(&pmpe_clip_workspace_size) lib_clip_workspace_size;
decltype(&pmpe_clip_grad_norm) lib_clip_grad_norm;
PyObject *g_error;         // PmpeError(code, what)
PyTypeObject *g_rms_norm;  // RmsNorm, a named tuple

struct Refused {
    int code;
    const char *what;
};
void want(bool ok, const char *what)
{
    if (!ok) throw Refused{PMPE_ERR_INVALID_ARG, what};
}
// No C++ exception leaves a function of this module: what it raises becomes a
// Python exception (PmpeError for refusals, PyTorch's own for its errors).
template <typename F> PyObject *guarded(F f)
{
    HANDLE_TH_ERRORS
    try {
        return f();
    } catch (const Refused &r) {
        PyObject *e = PyObject_CallFunction(g_error, "is", r.code, r.what);
        if (e) {
            PyErr_SetObject(g_error, e);
            Py_DECREF(e);
        }
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

const at::Tensor &tensor(PyObject *o, const char *what)
{
    want(THPVariable_Check(o), what);
    return THPVariable_Unpack(o);
}
// An optional argument: null for None.
const at::Tensor *optional(PyObject *o, const char *what) { return o == Py_None ? nullptr : &tensor(o, what); }
// The device that a call runs on, and its current stream.
struct Where {
    at::Device device;
    c10::cuda::CUDAGuard guard;
    explicit Where(const at::Tensor &t, const char *what) : device(checked(t, what)), guard(device) {}
    static at::Device checked(const at::Tensor &t, const char *what)
    {
        want(t.is_cuda(), what);
        return t.device();
    }
    void *stream() const { return c10::cuda::getCurrentCUDAStream(device.index()).stream(); }
};

int type_of(at::ScalarType t)
{
    return t == at::kFloat ? PMPE_F32 : t == at::kBFloat16 ? PMPE_BF16 : t == at::kHalf ? PMPE_F16 : -1;
}
bool is_vector(const at::Tensor &t, int64_t n, at::Device dev, at::ScalarType type)
{
    return t.scalar_type() == type && t.dim() == 1 && t.size(0) == n && t.device() == dev && t.is_contiguous();
}
bool is_matrix(const at::Tensor &t, int64_t rows, int64_t cols, at::Device dev, at::ScalarType type)
{
    return t.scalar_type() == type && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && t.device() == dev && t.is_contiguous();
}
// The type of a norm's weight: that of the rows or FP32.
int weight_type_of(const at::Tensor &w, int64_t H, at::Device dev, at::ScalarType type, const char *what)
{
    if (is_vector(w, H, dev, type)) return type_of(type);
    want(is_vector(w, H, dev, at::kFloat), what);
    return PMPE_F32;
}
// Elements from a row to the next (any value serves a single row); -1, which
// the library refuses, where a row's elements are not adjacent.
int64_t pitch(const at::Tensor &t)
{
    if (t.size(1) != 1 && t.stride(1) != 1) return -1;
    return t.size(0) > 1 ? t.stride(0) : t.size(1);
}
float narrow(double v) { return v > FLT_MAX ? INFINITY : v < -FLT_MAX ? -INFINITY : (float)v; }
int count(int64_t n)
{
    if (n > INT_MAX) throw Refused{PMPE_ERR_UNSUPPORTED_SHAPE, "more rows or columns than 32 bits count"};
    return (int)n;
}
at::Tensor empty(at::Device dev, at::ScalarType type, int64_t n) { return at::detail::empty_strided_cuda({n}, {1}, type, dev); }
at::Tensor empty(at::Device dev, at::ScalarType type, int64_t rows, int64_t cols)
{
    return at::detail::empty_strided_cuda({rows, cols}, {cols, 1}, type, dev);
}
// The library's call, which throws nothing, while other threads may run Python.
template <typename F> void run(const char *what, F f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    if (rc != PMPE_OK) throw Refused{rc, what};
}

// A caller's tensor was written to: autograd refuses a backward that saved it
// before.  (Tensors of inference mode have no versions.)
void written(const at::Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// A tuple (or a named one) of tensors; None where there is none.
PyObject *pack(PyTypeObject *type, std::initializer_list<at::Tensor> all)
{
    PyObject *t = type->tp_alloc(type, (Py_ssize_t)all.size());
    if (!t) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor &v : all) {
        PyObject *o = THPVariable_Wrap(v);  // None for an undefined tensor
        if (!o) {
            Py_DECREF(t);
            return nullptr;
        }
        PyTuple_SET_ITEM(t, i++, o);
    }
    return t;
}

void arguments(Py_ssize_t n, Py_ssize_t wanted) { want(n == wanted, "the number of arguments"); }

// (x, weight, residual, eps, quant, h_out)
PyObject *rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        arguments(n, 6);
        const at::Tensor &x = tensor(a[0], "rms_norm: x is a CUDA tensor"), &w = tensor(a[1], "rms_norm: weight is a tensor");
        const at::Tensor *res = optional(a[2], "rms_norm: residual is a tensor"), *h_out = optional(a[5], "rms_norm: h_out is a tensor");
        const double eps = PyFloat_AsDouble(a[3]);
        if (eps == -1. && PyErr_Occurred()) return nullptr;
        int quant = PMPE_QUANT_NONE;
        if (a[4] != Py_None) {
            const bool text = PyUnicode_Check(a[4]);
            quant = text && PyUnicode_CompareWithASCIIString(a[4], "block") == 0 ? PMPE_QUANT_BLOCK
                    : text && PyUnicode_CompareWithASCIIString(a[4], "row") == 0 ? PMPE_QUANT_ROW : -1;
            want(quant > 0, "rms_norm: quant is None, \"block\" or \"row\"");
        }
        pmpe_rms_norm_desc d = {};
        const at::ScalarType type = x.scalar_type();
        d.type = type_of(type);
        want(d.type >= 0 && x.dim() == 2, "rms_norm: x is [T, H] of FP32, BF16 or FP16");
        const int64_t T = x.size(0), H = x.size(1);
        d.T = count(T);
        d.H = count(H);
        d.weight_type = weight_type_of(w, H, x.device(), type, "rms_norm: weight is [H] of x's type or FP32, on x's device");
        const Where at(x, "rms_norm: x is a CUDA tensor");
        d.quant = quant;
        d.eps = narrow(eps);
        d.x = x.data_ptr();
        d.x_ld = pitch(x);
        d.weight = w.data_ptr();
        at::Tensor h;
        if (res) {
            want(res->scalar_type() == type && res->device() == at.device && res->dim() == 2 && res->size(0) == T && res->size(1) == H,
                 "rms_norm: residual is as x");
            want(!h_out || is_matrix(*h_out, T, H, at.device, type), "rms_norm: h_out is [T, H] of x's type without gaps");
            d.residual = res->data_ptr();
            d.residual_ld = pitch(*res);
            h = h_out ? *h_out : empty(at.device, type, T, H);
            d.h = h.data_ptr();
        } else {
            want(!h_out, "rms_norm: without a residual h is x");
            h = x;
        }
        const at::Tensor y = empty(at.device, quant ? at::kFloat8_e4m3fn : type, T, H);
        at::Tensor scale;
        if (quant) {
            scale = empty(at.device, at::kFloat, T, quant == PMPE_QUANT_BLOCK ? (H + 127) / 128 : 1);
            d.scale = (float *)scale.data_ptr();
        }
        const at::Tensor rstd = empty(at.device, at::kFloat, T);
        d.y = y.data_ptr();
        d.rstd = (float *)rstd.data_ptr();
        run("pmpe_rms_norm", [&, s = at.stream()] { return lib_rms_norm(&d, s); });
        if (h_out) written(*h_out);
        return pack(g_rms_norm, {y, scale, h, rstd});
    });
}

// (dy, h, weight, rstd, d_h, dx_dtype, need_dw)
PyObject *rms_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        arguments(n, 7);
        const at::Tensor &dy = tensor(a[0], "rms_norm_backward: dy is a tensor"), &h = tensor(a[1], "rms_norm_backward: h is a CUDA tensor"),
                         &w = tensor(a[2], "rms_norm_backward: weight is a tensor"), &rstd = tensor(a[3], "rms_norm_backward: rstd is a tensor");
        const at::Tensor *d_h = optional(a[4], "rms_norm_backward: d_h is a tensor");
        const int need_dw = PyObject_IsTrue(a[6]);
        if (need_dw < 0) return nullptr;
        pmpe_rms_norm_backward_desc d = {};
        const at::ScalarType type = h.scalar_type(), gt = dy.scalar_type();
        d.type = type_of(type);
        want(d.type >= 0 && h.dim() == 2 && h.is_contiguous(), "rms_norm_backward: h is [T, H] of FP32, BF16 or FP16 without gaps");
        const int64_t T = h.size(0), H = h.size(1);
        d.T = count(T);
        d.H = count(H);
        d.weight_type = weight_type_of(w, H, h.device(), type, "rms_norm_backward: weight is [H] of h's type or FP32, on h's device");
        const Where at(h, "rms_norm_backward: h is a CUDA tensor");
        at::ScalarType xt = type;
        if (a[5] != Py_None) {
            want(THPDtype_Check(a[5]), "rms_norm_backward: dx_dtype is a dtype");
            xt = ((THPDtype *)a[5])->scalar_type;
        }
        want(xt == type || xt == at::kFloat, "rms_norm_backward: dx is of h's type or FP32");
        want((gt == type || gt == at::kFloat) && is_matrix(dy, T, H, at.device, gt), "rms_norm_backward: dy is [T, H] of h's type or FP32 without gaps");
        want(is_vector(rstd, T, at.device, at::kFloat), "rms_norm_backward: rstd is FP32 [T]");
        want(!d_h || is_matrix(*d_h, T, H, at.device, xt), "rms_norm_backward: d_h is [T, H] of dx's type without gaps");
        d.dy_type = type_of(gt);
        d.dx_type = type_of(xt);
        d.dy = dy.data_ptr();
        d.h = h.data_ptr();
        d.weight = w.data_ptr();
        d.rstd = (const float *)rstd.data_ptr();
        d.d_h = d_h ? d_h->data_ptr() : nullptr;
        const at::Tensor dx = empty(at.device, xt, T, H);
        d.dx = dx.data_ptr();
        at::Tensor dw, ws;
        if (need_dw) {
            d.workspace_bytes = lib_rms_norm_backward_workspace_size(d.T, d.H);
            dw = empty(at.device, at::kFloat, H);
            ws = empty(at.device, at::kByte, (int64_t)d.workspace_bytes);
            d.dw = (float *)dw.data_ptr();
            d.workspace = ws.data_ptr();
        }
        run("pmpe_rms_norm_backward", [&, s = at.stream()] { return lib_rms_norm_backward(&d, s); });
        return pack(&PyTuple_Type, {dx, dw});
    });
}

// (E_pub, E_priv, k, score, renormalize, groups, top_groups, groups_priv,
// top_groups_priv, group_score, scale): the descriptor of a router as bytes,
// once the library has taken it for a batch of no tokens.
PyObject *router(PyObject *, PyObject *args)
{
    return guarded([&]() -> PyObject * {
        pmpe_route_desc d = {};
        if (!PyArg_ParseTuple(args, "iiiiiiiiiif", &d.E_pub, &d.E_priv, &d.k, &d.score, &d.renormalize, &d.groups_pub, &d.top_groups_pub,
                              &d.groups_priv, &d.top_groups_priv, &d.group_score, &d.scale))
            return nullptr;
        d.ld = (int64_t)d.E_pub + d.E_priv;
        run("pmpe_route", [&] { return lib_route(&d, nullptr); });
        return PyBytes_FromStringAndSize((const char *)&d, sizeof(d));
    });
}

// The descriptor of a call: the router's, with the logits and the policy.
pmpe_route_desc route_desc(PyObject *desc, const at::Tensor &logits, const at::Tensor *policy, at::Device dev)
{
    pmpe_route_desc d;
    want(PyBytes_Check(desc) && PyBytes_GET_SIZE(desc) == (Py_ssize_t)sizeof(d), "Router: its descriptor");
    memcpy(&d, PyBytes_AS_STRING(desc), sizeof(d));
    d.logits_type = type_of(logits.scalar_type());
    want(d.logits_type >= 0 && logits.dim() == 2 && logits.size(1) == d.ld, "Router: logits are [T, E] of FP32, BF16 or FP16");
    d.T = count(logits.size(0));
    d.ld = pitch(logits);
    d.logits = logits.data_ptr();
    want(!policy || is_vector(*policy, d.T, dev, at::kByte), "Router: policy is uint8 [T] on the logits' device");
    d.policy = policy ? (const uint8_t *)policy->data_ptr() : nullptr;
    return d;
}

// (descriptor, logits, policy, bias, load)
PyObject *route(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        arguments(n, 5);
        const at::Tensor &logits = tensor(a[1], "Router: logits are a CUDA tensor");
        const at::Tensor *policy = optional(a[2], "Router: policy is a tensor"), *bias = optional(a[3], "Router: bias is a tensor"),
                         *load = optional(a[4], "Router: load is a tensor");
        const Where at(logits, "Router: logits are a CUDA tensor");
        pmpe_route_desc d = route_desc(a[0], logits, policy, at.device);
        const int64_t E = (int64_t)d.E_pub + d.E_priv;
        want(!bias || is_vector(*bias, E, at.device, at::kFloat), "Router: bias is FP32 [E] on the logits' device");
        want(!load || is_vector(*load, E, at.device, at::kInt), "Router: load is int32 [E] on the logits' device");
        const at::Tensor idx = empty(at.device, at::kInt, d.T, d.k), w = empty(at.device, at::kFloat, d.T, d.k);
        d.bias = bias ? (const float *)bias->data_ptr() : nullptr;
        d.load = load ? (int32_t *)load->data_ptr() : nullptr;
        d.topk_idx = (int32_t *)idx.data_ptr();
        d.topk_w = (float *)w.data_ptr();
        run("pmpe_route", [&, s = at.stream()] { return lib_route(&d, s); });
        if (load) written(*load);
        return pack(&PyTuple_Type, {idx, w});
    });
}

// (descriptor, logits, policy, idx, dw)
PyObject *route_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        arguments(n, 5);
        const at::Tensor &logits = tensor(a[1], "Router: logits are a CUDA tensor");
        const at::Tensor *policy = optional(a[2], "Router: policy is a tensor");
        const at::Tensor &idx = tensor(a[3], "Router: idx is a tensor"), &dw = tensor(a[4], "Router: dw is a tensor");
        const Where at(logits, "Router: logits are a CUDA tensor");
        pmpe_route_desc d = route_desc(a[0], logits, policy, at.device);
        want(is_matrix(idx, d.T, d.k, at.device, at::kInt), "Router: idx is int32 [T, k] on the logits' device");
        want(is_matrix(dw, d.T, d.k, at.device, at::kFloat), "Router: dw is FP32 [T, k] on the logits' device");
        const at::Tensor d_logits = empty(at.device, logits.scalar_type(), d.T, (int64_t)d.E_pub + d.E_priv);
        d.topk_idx = (int32_t *)idx.data_ptr();
        run("pmpe_route_backward", [&d, from = (const float *)dw.data_ptr(), to = d_logits.data_ptr(), s = at.stream()] {
            return lib_route_backward(&d, from, to, s);
        });
        return THPVariable_Wrap(d_logits);
    });
}

// Whether the tensor's elements fill a run of memory, in some order.
bool dense(const at::Tensor &t)
{
    std::vector<std::pair<int64_t, int64_t>> dims;
    for (int64_t i = 0; i < t.dim(); ++i)
        if (t.size(i) != 1) dims.emplace_back(t.stride(i), t.size(i));
    std::sort(dims.begin(), dims.end());
    int64_t next = 1;
    for (const auto &d : dims) {
        if (d.first != next) return false;
        next *= d.second;
    }
    return true;
}

// (gradients, max_norm, outputs or None): a list or tuple each
PyObject *clip_grad_norm(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> PyObject * {
        arguments(n_args, 3);
        const double max_norm = PyFloat_AsDouble(a[1]);
        if (max_norm == -1. && PyErr_Occurred()) return nullptr;
        auto is_list = [](PyObject *o) { return PyList_Check(o) || PyTuple_Check(o); };
        want(is_list(a[0]) && (a[2] == Py_None || is_list(a[2])), "clip_grad_norm: gradients are a list or a dict of tensors");
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
        const bool apart = a[2] != Py_None;  // outputs of their own (an empty list's items are null)
        want(n > 0 && (!apart || PySequence_Fast_GET_SIZE(a[2]) == n), "clip_grad_norm: gradients, and an output for each or none, are wanted");
        PyObject **g = PySequence_Fast_ITEMS(a[0]), **o = apart ? PySequence_Fast_ITEMS(a[2]) : nullptr;
        const Where at(tensor(g[0], "clip_grad_norm: gradients are CUDA tensors"), "clip_grad_norm: gradients are CUDA tensors");
        std::vector<pmpe_grad> grads((size_t)count(n));
        std::vector<at::Tensor> outputs;  // held: the lists may change while other threads run
        outputs.reserve((size_t)n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            const at::Tensor &t = tensor(g[i], "clip_grad_norm: gradients are CUDA tensors");
            pmpe_grad &q = grads[(size_t)i];
            q.type = type_of(t.scalar_type());
            want(q.type >= 0 && t.device() == at.device, "clip_grad_norm: gradients are FP32, BF16 or FP16 tensors of one device");
            q.n = t.numel();
            q.grad = q.out = t.data_ptr();
            bool whole = t.is_contiguous();
            if (o) {
                const at::Tensor &u = tensor(o[i], "clip_grad_norm: outputs are CUDA tensors");
                want(u.scalar_type() == t.scalar_type() && u.device() == at.device && u.numel() == q.n,
                     "clip_grad_norm: outputs are of their gradients' types and sizes");
                q.out = u.data_ptr();
                if (!whole || !u.is_contiguous()) {
                    want(u.sizes() == t.sizes() && u.strides() == t.strides(), "clip_grad_norm: an output is in another order than its gradient");
                    whole = false;
                }
            }
            want(whole || dense(t), "clip_grad_norm: a gradient has gaps");
            outputs.push_back(o ? tensor(o[i], "clip_grad_norm: outputs are CUDA tensors") : t);
        }
        const size_t bytes = lib_clip_workspace_size((int)n);
        const at::Tensor norm = at::detail::empty_strided_cuda({}, {}, at::kFloat, at.device), ws = empty(at.device, at::kByte, (int64_t)bytes);
        run("pmpe_clip_grad_norm", [&, to = (float *)norm.data_ptr(), scratch = ws.data_ptr(), s = at.stream()] {
            return lib_clip_grad_norm(grads.data(), (int)n, narrow(max_norm), to, scratch, bytes, s);
        });
        if (apart || max_norm < INFINITY)  // else the norm alone
            for (const at::Tensor &t : outputs) written(t);
        return THPVariable_Wrap(norm);
    });
}

// (PmpeError, RmsNorm, the library's functions' addresses in the order above)
PyObject *setup(PyObject *, PyObject *args)
{
    unsigned long long f[7];
    PyObject *error, *norm;
    if (!PyArg_ParseTuple(args, "OO!KKKKKKK", &error, &PyType_Type, &norm, f, f + 1, f + 2, f + 3, f + 4, f + 5, f + 6)) return nullptr;
    Py_INCREF(error);
    Py_INCREF(norm);
    g_error = error;
    g_rms_norm = (PyTypeObject *)norm;
    lib_rms_norm = (decltype(lib_rms_norm))f[0];
    lib_rms_norm_backward_workspace_size = (decltype(lib_rms_norm_backward_workspace_size))f[1];
    lib_rms_norm_backward = (decltype(lib_rms_norm_backward))f[2];
    lib_route = (decltype(lib_route))f[3];
    lib_route_backward = (decltype(lib_route_backward))f[4];
    lib_clip_workspace_size = (decltype(lib_clip_workspace_size))f[5];
    lib_clip_grad_norm = (decltype(lib_clip_grad_norm))f[6];
    Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void *)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(rms_norm), FAST(rms_norm_backward), FAST(route), FAST(route_backward), FAST(clip_grad_norm),
                         {"router", router, METH_VARARGS, nullptr}, {"setup", setup, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, methods};

}  // namespace

// built_for: the PyTorch whose headers this was compiled with.
PyMODINIT_FUNC PyInit__ops()
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", PMPE_BUILT_FOR) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
