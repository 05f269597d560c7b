// Short way into the calls of block.py whose kernels take less time than Python takes to describe their arguments: a single
// token's convolution and scan, and the projections.  Each function checks what block.py checks and, where everything is in its ordinary
// place (the arguments' types, shapes, contiguity, one CUDA device, the current stream), fills the record, makes the call and
// returns the output; otherwise it returns None and block.py goes its own way, which also says what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/ttc_block.h"

namespace {

decltype(&ttc_causal_conv_step) conv_step_call;
decltype(&ttc_selective_scan_step) scan_step_call;
decltype(&ttc_linear) linear_call;
decltype(&ttc_linear_workspace) linear_workspace_call;

// A tensor argument: absent (None), present, or something else.
struct Arg {
    const at::Tensor* t = nullptr;
    bool ok = true;
    explicit Arg(PyObject* o)
    {
        if (o == Py_None)
            return;
        ok = THPVariable_Check(o);
        if (ok)
            t = &THPVariable_Unpack(o);
    }
    void* ptr() const { return t ? t->data_ptr() : nullptr; }
};

int type_code(at::ScalarType t)
{
    return t == at::kFloat ? TTC_F32 : t == at::kBFloat16 ? TTC_BF16 : t == at::kHalf ? TTC_F16 : -1;
}

bool here(const at::Tensor& t, at::ScalarType type, c10::Device device) { return t.scalar_type() == type && t.device() == device; }

// a contiguous tensor of that shape, or none
bool dense(const Arg& a, at::IntArrayRef shape, at::ScalarType type, c10::Device device)
{
    return a.ok && (!a.t || (here(*a.t, type, device) && a.t->sizes() == shape && a.t->is_contiguous()));
}

// rows [batch][channels] of contiguous channels, or none
bool rows(const Arg& a, int64_t batch, int64_t channels, at::ScalarType type, c10::Device device, ttc_rows& r)
{
    r = ttc_rows{nullptr, 0, 0};
    if (!a.ok || !a.t)
        return a.ok;
    const at::Tensor& t = *a.t;
    if (!here(t, type, device) || t.dim() != 2 || t.size(0) != batch || t.size(1) != channels || (channels > 1 && t.stride(1) != 1))
        return false;
    r = ttc_rows{t.data_ptr(), t.stride(0), 0};
    return true;
}

// rows of B or C: [batch][n] or [batch][groups][n]
bool shared_rows(const at::Tensor& t, int64_t batch, int64_t groups, int64_t n, at::ScalarType type, c10::Device device, ttc_rows& r)
{
    const int64_t k = t.dim();
    if (!here(t, type, device) || (k != 2 && k != 3) || t.size(0) != batch || t.size(k - 1) != n || (n > 1 && t.stride(k - 1) != 1))
        return false;
    if (k == 2 ? groups != 1 : t.size(1) != groups || (groups > 1 && t.stride(1) != n))
        return false;
    r = ttc_rows{t.data_ptr(), t.stride(0), 0};
    return true;
}

PyObject* give(PyObject* y_arg, const at::Tensor& y)
{
    if (y_arg != Py_None) {
        Py_INCREF(y_arg);
        return y_arg;
    }
    return THPVariable_Wrap(y);
}

// (x, w, state, bias, act, y)
PyObject* conv_step(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 6 || !conv_step_call)
        Py_RETURN_NONE;
    try {
        const Arg x(args[0]), w(args[1]), state(args[2]), bias(args[3]), y_arg(args[5]);
        const long act = PyLong_AsLong(args[4]);
        if (!x.t || !w.t || !state.t || !bias.ok || !y_arg.ok || act < 0 || PyErr_Occurred())
            return PyErr_Clear(), Py_NewRef(Py_None);
        const at::Tensor& xt = *x.t;
        if (!xt.is_cuda() || xt.dim() != 2 || w.t->dim() != 2)
            Py_RETURN_NONE;
        const auto type = xt.scalar_type();
        const auto device = xt.device();
        const int64_t batch = xt.size(0), d = xt.size(1), taps = w.t->size(1);
        ttc_conv_args a = {};
        if (type_code(type) < 0 || batch == 0 || d >= INT32_MAX || taps < 2 || taps > 4 || !dense(w, {d, taps}, at::kFloat, device) ||
            !dense(bias, {d}, at::kFloat, device) || !dense(state, {batch, taps - 1, d}, type, device) || !rows(x, batch, d, type, device, a.x))
            Py_RETURN_NONE;
        at::Tensor y;
        if (!y_arg.t)
            y = at::empty_like(xt);
        if (!rows(y_arg.t ? y_arg : x, batch, d, type, device, a.y))
            Py_RETURN_NONE;
        if (!y_arg.t)
            a.y = ttc_rows{y.data_ptr(), y.stride(0), 0};
        a.batch = batch;
        a.tokens = 1;
        a.d = (int32_t)d;
        a.taps = (int32_t)taps;
        a.act = (int32_t)act;
        a.dtype = type_code(type);
        a.w = static_cast<const float*>(w.ptr());
        a.bias = static_cast<const float*>(bias.ptr());
        a.state_out = state.ptr();
        if (conv_step_call(device.index(), &a, c10::cuda::getCurrentCUDAStream(device.index()).stream()) != TTC_OK)
            Py_RETURN_NONE;
        return give(args[5], y);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// (x, delta, A, B, C, state, D, z, delta_bias, softplus, y)
PyObject* scan_step(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 11 || !scan_step_call)
        Py_RETURN_NONE;
    try {
        const Arg x(args[0]), delta(args[1]), A(args[2]), B(args[3]), C(args[4]), state(args[5]), D(args[6]), z(args[7]), bias(args[8]), y_arg(args[10]);
        const int softplus = PyObject_IsTrue(args[9]);
        if (!x.t || !delta.t || !A.t || !B.t || !C.t || !state.t || !D.ok || !z.ok || !bias.ok || !y_arg.ok || softplus < 0)
            return PyErr_Clear(), Py_NewRef(Py_None);
        const at::Tensor& xt = *x.t;
        if (!xt.is_cuda() || xt.dim() != 2 || A.t->dim() != 2 || (B.t->dim() != 2 && B.t->dim() != 3))
            Py_RETURN_NONE;
        const auto type = xt.scalar_type();
        const auto device = xt.device();
        const int64_t batch = xt.size(0), d = xt.size(1), n = A.t->size(1), groups = B.t->dim() == 3 ? B.t->size(1) : 1;
        ttc_scan_args a = {};
        if (type_code(type) < 0 || batch == 0 || d >= INT32_MAX || n >= INT32_MAX || groups >= INT32_MAX || !dense(A, {d, n}, at::kFloat, device) ||
            !dense(D, {d}, at::kFloat, device) || !dense(bias, {d}, at::kFloat, device) || !dense(state, {batch, d, n}, at::kFloat, device) ||
            !rows(x, batch, d, type, device, a.x) || !rows(delta, batch, d, type, device, a.delta) || !rows(z, batch, d, type, device, a.z) ||
            !shared_rows(*B.t, batch, groups, n, type, device, a.B) || !shared_rows(*C.t, batch, groups, n, type, device, a.C))
            Py_RETURN_NONE;
        at::Tensor y;
        if (y_arg.t) {
            if (!rows(y_arg, batch, d, type, device, a.y))
                Py_RETURN_NONE;
        } else {
            y = at::empty_like(xt);
            a.y = ttc_rows{y.data_ptr(), y.stride(0), 0};
        }
        a.batch = batch;
        a.tokens = 1;
        a.d = (int32_t)d;
        a.n = (int32_t)n;
        a.groups = (int32_t)groups;
        a.dtype = type_code(type);
        a.softplus = softplus;
        a.A = static_cast<const float*>(A.ptr());
        a.D = static_cast<const float*>(D.ptr());
        a.delta_bias = static_cast<const float*>(bias.ptr());
        a.state_out = static_cast<float*>(state.ptr());
        if (scan_step_call(device.index(), &a, c10::cuda::getCurrentCUDAStream(device.index()).stream()) != TTC_OK)
            Py_RETURN_NONE;
        return give(args[10], y);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// (x, w, bias, act, residual, y, float32 output): rows [rows][k] with one stride, no scratch
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 7 || !linear_call || !linear_workspace_call)
        Py_RETURN_NONE;
    try {
        const Arg x(args[0]), w(args[1]), bias(args[2]), residual(args[4]), y_arg(args[5]);
        const long act = PyLong_AsLong(args[3]);
        const int wide = PyObject_IsTrue(args[6]);
        if (!x.t || !w.t || !bias.ok || !residual.ok || !y_arg.ok || act < 0 || wide < 0 || PyErr_Occurred())
            return PyErr_Clear(), Py_NewRef(Py_None);
        const at::Tensor &xt = *x.t, &wt = *w.t;
        const auto type = xt.scalar_type();
        const auto device = xt.device();
        if (!xt.is_cuda() || xt.dim() != 2 || wt.dim() != 2 || (type != at::kBFloat16 && type != at::kHalf))
            Py_RETURN_NONE;
        const auto out = wide ? at::kFloat : type;
        const int64_t n = xt.size(0), k = xt.size(1), m = wt.size(0);
        ttc_rows xr, wr, rr, yr;
        if (n == 0 || k >= INT32_MAX || m >= INT32_MAX || !dense(bias, {m}, at::kFloat, device) || !rows(x, n, k, type, device, xr) ||
            !rows(w, m, k, type, device, wr) || !rows(residual, n, m, out, device, rr))
            Py_RETURN_NONE;
        ttc_linear_args a = {};
        a.rows = n;
        a.k = (int32_t)k;
        a.m = (int32_t)m;
        a.dtype = type_code(type);
        a.out_dtype = type_code(out);
        a.act = (int32_t)act;
        a.x = xr.ptr, a.ldx = xr.bstride;
        a.w = wr.ptr, a.ldw = wr.bstride;
        a.bias = static_cast<const float*>(bias.ptr());
        a.residual = rr.ptr, a.ldr = rr.bstride;
        at::Tensor y;
        if (y_arg.t) {
            if (!rows(y_arg, n, m, out, device, yr))
                Py_RETURN_NONE;
            a.y = yr.ptr, a.ldy = yr.bstride;
        } else {
            y = at::empty({n, m}, xt.options().dtype(out));
            a.y = y.data_ptr(), a.ldy = m;
        }
        const int64_t need = linear_workspace_call(device.index(), &a);
        if (need < 0)
            Py_RETURN_NONE;
        at::Tensor ws;
        if (need > 0)
            ws = at::empty({need}, xt.options().dtype(at::kByte));
        if (linear_call(device.index(), &a, need ? ws.data_ptr() : nullptr, need, c10::cuda::getCurrentCUDAStream(device.index()).stream()) != TTC_OK)
            Py_RETURN_NONE;
        return give(args[5], y);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// Addresses of the library's functions, in the order of the declarations above, and the sizes of the records that they take (a module
// that was compiled with another header than the library must not fill them).
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 7) {
        PyErr_SetString(PyExc_TypeError, "bind takes four addresses and three sizes");
        return nullptr;
    }
    void* at[4];
    for (int i = 0; i < 4; ++i) {
        at[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred())
            return nullptr;
    }
    const long sizes[3] = {(long)sizeof(ttc_conv_args), (long)sizeof(ttc_scan_args), (long)sizeof(ttc_linear_args)};
    for (int i = 0; i < 3; ++i) {
        const long size = PyLong_AsLong(args[4 + i]);
        if (PyErr_Occurred())
            return nullptr;
        if (size != sizes[i]) {
            PyErr_Format(PyExc_ImportError, "_step.so was built for records of %ld bytes, not %ld: build it again", sizes[i], size);
            return nullptr;
        }
    }
    conv_step_call = reinterpret_cast<decltype(conv_step_call)>(at[0]);
    scan_step_call = reinterpret_cast<decltype(scan_step_call)>(at[1]);
    linear_call = reinterpret_cast<decltype(linear_call)>(at[2]);
    linear_workspace_call = reinterpret_cast<decltype(linear_workspace_call)>(at[3]);
    Py_RETURN_NONE;
}

#define TTC_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {TTC_METHOD(bind), TTC_METHOD(conv_step), TTC_METHOD(scan_step), TTC_METHOD(linear), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_step", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__step(void) { return PyModule_Create(&module); }
