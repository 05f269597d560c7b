// Short way into the calls of block.py whose kernels take less time than Python takes to describe their arguments: a single
// token's convolution, scan and linear attention, linear attention and the norms with their gradients, and the projections.  Each function checks what block.py checks and, where everything is in its ordinary
// place (the arguments' types, shapes, contiguity, one CUDA device, the current stream), fills the record, makes the call and
// returns the output; otherwise it returns None and block.py goes its own way, which also says what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/ttc_block.h"

namespace {

decltype(&ttc_causal_conv_step) conv_step_call;
decltype(&ttc_selective_scan_step) scan_step_call;
decltype(&ttc_linear) linear_call;
decltype(&ttc_linear_workspace) linear_workspace_call;
decltype(&ttc_decay_attention) attention_call;
decltype(&ttc_decay_attention_workspace) attention_workspace_call;
decltype(&ttc_decay_attention_step) attention_step_call;
decltype(&ttc_block_norm) norm_call;
decltype(&ttc_decay_attention_grad) attention_grad_call;
decltype(&ttc_decay_attention_grad_workspace) attention_grad_workspace_call;
decltype(&ttc_block_norm_grad) norm_grad_call;
decltype(&ttc_block_norm_grad_workspace) norm_grad_workspace_call;

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

// rows of heads [lead..][heads][width], the heads one behind the other; `lead` is the number of dimensions in front (2: batch and tokens)
bool head_rows(const at::Tensor& t, const at::Tensor& like, int lead, int64_t heads, int64_t width, bool packed, ttc_rows& r)
{
    if (!here(t, like.scalar_type(), like.device()) || t.dim() != lead + 2 || t.size(lead) != heads || t.size(lead + 1) != width ||
        (width > 1 && t.stride(lead + 1) != 1) || (heads > 1 && t.stride(lead) != width))
        return false;
    for (int i = 0; i < lead; ++i)
        if (t.size(i) != like.size(i))
            return false;
    r = lead == 2 ? ttc_rows{t.data_ptr(), t.stride(0), t.stride(1)} : packed ? ttc_rows{t.data_ptr(), 0, t.stride(0)} : ttc_rows{t.data_ptr(), t.stride(0), 0};
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

// What a call of linear attention is given, checked; the record without y and state_out.
struct Attention {
    Arg q, k, v, A, delta, bias, state, offsets;
    ttc_decay_args a = {};
    int lead = 0;
    bool packed = false, ok = false;
    // args: (q, k, v, A, delta, delta_bias, softplus, scale or None, state, offsets)
    Attention(PyObject* const* args, bool step)
        : q(args[0]), k(args[1]), v(args[2]), A(args[3]), delta(args[4]), bias(args[5]), state(args[8]), offsets(args[9])
    {
        const int softplus = PyObject_IsTrue(args[6]);
        if (!q.t || !k.t || !v.t || !A.t || !delta.ok || !bias.ok || !state.ok || !offsets.ok || softplus < 0 || (bias.t && !delta.t))
            return;
        const at::Tensor& vt = *v.t;
        const auto type = vt.scalar_type();
        const auto device = vt.device();
        packed = offsets.t;
        lead = step || packed ? 1 : 2;
        if (!vt.is_cuda() || (type != at::kBFloat16 && type != at::kHalf) || vt.dim() != lead + 2 || q.t->dim() != lead + 2 || (step && packed))
            return;
        const int64_t heads = vt.size(lead), dv = vt.size(lead + 1), groups = q.t->size(lead), dk = q.t->size(lead + 1);
        int64_t batch = vt.size(0);
        const int64_t tokens = step ? 1 : packed ? vt.size(0) : vt.size(1);
        if (packed) {
            if (!here(*offsets.t, at::kInt, device) || offsets.t->dim() != 1 || offsets.t->size(0) < 1 || !offsets.t->is_contiguous())
                return;
            batch = offsets.t->size(0) - 1;
        }
        if (batch == 0 || tokens == 0 || heads >= INT32_MAX || groups >= INT32_MAX || dk < 1 || dk > 128 || dv > 128 || !dense(A, {heads}, at::kFloat, device) ||
            !dense(bias, {heads}, at::kFloat, device) || !dense(state, {batch, heads, dk, dv}, at::kFloat, device) || !head_rows(*q.t, vt, lead, groups, dk, packed, a.q) ||
            !head_rows(*k.t, vt, lead, groups, dk, packed, a.k) || !head_rows(vt, vt, lead, heads, dv, packed, a.v))
            return;
        if (delta.t) {                           // [lead..][heads]
            const at::Tensor& t = *delta.t;
            if (!here(t, type, device) || t.dim() != lead + 1 || t.size(lead) != heads || (heads > 1 && t.stride(lead) != 1) || t.size(0) != vt.size(0) ||
                (lead == 2 && t.size(1) != vt.size(1)))
                return;
            a.delta = token_rows(t);
        }
        double scale = 1.0 / std::sqrt((double)dk);
        if (args[7] != Py_None) {
            scale = PyFloat_AsDouble(args[7]);
            if (PyErr_Occurred())
                return;
        }
        a.batch = batch;
        a.tokens = tokens;
        a.seq_offsets = packed ? static_cast<const int32_t*>(offsets.ptr()) : nullptr;
        a.heads = (int32_t)heads;
        a.groups = (int32_t)groups;
        a.dk = (int32_t)dk;
        a.dv = (int32_t)dv;
        a.dtype = type_code(type);
        a.softplus = softplus;
        a.scale = (float)scale;
        a.A = static_cast<const float*>(A.ptr());
        a.delta_bias = static_cast<const float*>(bias.ptr());
        a.state = static_cast<const float*>(state.ptr());
        ok = true;
    }
    ttc_rows token_rows(const at::Tensor& t) const
    {
        return lead == 2 ? ttc_rows{t.data_ptr(), t.stride(0), t.stride(1)} : packed ? ttc_rows{t.data_ptr(), 0, t.stride(0)} : ttc_rows{t.data_ptr(), t.stride(0), 0};
    }
};

PyObject* none()
{
    PyErr_Clear();
    return Py_NewRef(Py_None);
}

// (q, k, v, A, delta, delta_bias, softplus, scale or None, state, offsets, y, state_out, step)
PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 13 || !attention_call)
        Py_RETURN_NONE;
    try {
        const int step = PyObject_IsTrue(args[12]);
        if (step < 0)
            return none();
        Attention c(args, step);
        const Arg y_arg(args[10]), state_out(args[11]);
        if (!c.ok || !y_arg.ok)
            return none();
        const at::Tensor& vt = *c.v.t;
        ttc_decay_args& a = c.a;
        const auto device = vt.device();
        if (!dense(state_out, {a.batch, a.heads, a.dk, a.dv}, at::kFloat, device))
            return none();
        at::Tensor y;
        if (!y_arg.t)
            y = at::empty(vt.sizes(), vt.options());
        if (!head_rows(y_arg.t ? *y_arg.t : y, vt, c.lead, a.heads, a.dv, c.packed, a.y))
            return none();
        a.state_out = static_cast<float*>(state_out.ptr());
        void* stream = c10::cuda::getCurrentCUDAStream(device.index()).stream();
        if (step) {
            if (attention_step_call(device.index(), &a, stream) != TTC_OK)
                return none();
            return give(args[10], y);
        }
        const int64_t need = attention_workspace_call(device.index(), &a);
        if (need < 0)
            return none();
        at::Tensor ws;
        if (need > 0)
            ws = at::empty({need}, vt.options().dtype(at::kByte));
        if (attention_call(device.index(), &a, need ? ws.data_ptr() : nullptr, need, stream) != TTC_OK)
            return none();
        return give(args[10], y);
    } catch (...) {
        return none();
    }
}

// Puts a tensor into a dict; false on failure.
bool put(PyObject* d, const char* name, const at::Tensor& t)
{
    PyObject* o = THPVariable_Wrap(t);
    const bool ok = o && PyDict_SetItemString(d, name, o) == 0;
    Py_XDECREF(o);
    return ok;
}

// (q, k, v, A, delta, delta_bias, softplus, scale or None, state, offsets, dy, dstate_out): a dict of all gradients
PyObject* attention_grad(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 12 || !attention_grad_call)
        Py_RETURN_NONE;
    try {
        Attention c(args, false);
        const Arg dy(args[10]), dlast(args[11]);
        if (!c.ok || !dy.t)
            return none();
        const at::Tensor &vt = *c.v.t, &qt = *c.q.t;
        const ttc_decay_args& a = c.a;
        const auto device = vt.device();
        ttc_decay_grads g = {};
        if (!dense(dlast, {a.batch, a.heads, a.dk, a.dv}, at::kFloat, device) || !head_rows(*dy.t, vt, c.lead, a.heads, a.dv, c.packed, g.dy))
            return none();
        const auto f32 = vt.options().dtype(at::kFloat);
        const at::Tensor dq = at::empty(qt.sizes(), vt.options()), dk = at::empty(qt.sizes(), vt.options()), dv = at::empty(vt.sizes(), vt.options()), dA = at::empty({a.heads}, f32),
                         dstate = at::empty({a.batch, a.heads, a.dk, a.dv}, f32);
        at::Tensor ddelta, dbias;
        head_rows(dq, vt, c.lead, a.groups, a.dk, c.packed, g.dq);
        head_rows(dk, vt, c.lead, a.groups, a.dk, c.packed, g.dk);
        head_rows(dv, vt, c.lead, a.heads, a.dv, c.packed, g.dv);
        g.dA = static_cast<float*>(dA.data_ptr());
        g.dstate = static_cast<float*>(dstate.data_ptr());
        g.dstate_out = static_cast<const float*>(dlast.ptr());
        if (c.delta.t) {
            ddelta = at::empty(c.delta.t->sizes(), vt.options());
            dbias = at::empty({a.heads}, f32);
            g.ddelta = c.token_rows(ddelta);
            g.ddelta_bias = static_cast<float*>(dbias.data_ptr());
        }
        const int64_t need = attention_grad_workspace_call(device.index(), &a, &g);
        if (need < 0)
            return none();
        at::Tensor ws;
        if (need > 0)
            ws = at::empty({need}, vt.options().dtype(at::kByte));
        if (attention_grad_call(device.index(), &a, &g, need ? ws.data_ptr() : nullptr, need, c10::cuda::getCurrentCUDAStream(device.index()).stream()) != TTC_OK)
            return none();
        PyObject* d = PyDict_New();
        if (!d || !put(d, "dq", dq) || !put(d, "dk", dk) || !put(d, "dv", dv) || (c.delta.t && !put(d, "ddelta", ddelta)) || !put(d, "dA", dA) ||
            (c.delta.t && !put(d, "ddelta_bias", dbias)) || !put(d, "dstate", dstate)) {
            Py_XDECREF(d);
            return none();
        }
        return d;
    } catch (...) {
        return none();
    }
}

// rows of d channels with one stride, whatever their leading dimensions (contiguous ones are taken together), or none
bool flat_rows(const Arg& a, const at::Tensor& like, const void*& ptr, int64_t& ld)
{
    ptr = nullptr, ld = 0;
    if (!a.ok || !a.t)
        return a.ok;
    const at::Tensor& t = *a.t;
    if (!here(t, like.scalar_type(), like.device()) || t.sizes() != like.sizes())
        return false;
    const int64_t d = t.size(t.dim() - 1);
    if (t.is_contiguous())
        ld = d;
    else if (t.dim() == 2 && (d <= 1 || t.stride(1) == 1) && t.stride(0) >= d)
        ld = t.stride(0);
    else
        return false;
    ptr = t.data_ptr();
    return true;
}

// (x, w_post, z, scale, residual, w_pre, eps, groups, h, y): the pair (h, y)
PyObject* norm(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 10 || !norm_call)
        Py_RETURN_NONE;
    try {
        const Arg x(args[0]), w_post(args[1]), z(args[2]), scale(args[3]), residual(args[4]), w_pre(args[5]), h_arg(args[8]), y_arg(args[9]);
        const double eps = PyFloat_AsDouble(args[6]);
        const long groups = PyErr_Occurred() ? -1 : PyLong_AsLong(args[7]);
        if (PyErr_Occurred() || !x.t || !z.ok || !residual.ok || !h_arg.ok || !y_arg.ok || groups < 1 || groups >= INT32_MAX)
            return PyErr_Clear(), Py_NewRef(Py_None);
        const at::Tensor& xt = *x.t;
        const bool changed = w_post.t || z.t || scale.t || residual.t;
        if (!xt.is_cuda() || xt.dim() < 1 || type_code(xt.scalar_type()) < 0 || xt.numel() == 0 || (!changed && !w_pre.t) || (y_arg.t && !w_pre.t))
            Py_RETURN_NONE;
        const int64_t d = xt.size(xt.dim() - 1);
        const auto device = xt.device();
        ttc_norm_args a = {};
        const void *h_ptr, *y_ptr;
        if (d >= INT32_MAX || !dense(w_post, {d}, at::kFloat, device) || !dense(scale, {d}, at::kFloat, device) || !dense(w_pre, {d}, at::kFloat, device) ||
            !flat_rows(x, xt, a.x, a.ldx) || !flat_rows(z, xt, a.z, a.ldz) || !flat_rows(residual, xt, a.residual, a.ldr) || !flat_rows(h_arg, xt, h_ptr, a.ldh) ||
            !flat_rows(y_arg, xt, y_ptr, a.ldy))
            Py_RETURN_NONE;
        at::Tensor h, y;
        if (changed && !h_arg.t) {
            h = at::empty(xt.sizes(), xt.options());
            h_ptr = h.data_ptr(), a.ldh = d;
        }
        if (w_pre.t && !y_arg.t) {
            y = at::empty(xt.sizes(), xt.options());
            y_ptr = y.data_ptr(), a.ldy = d;
        }
        a.rows = xt.numel() / d;
        a.d = (int32_t)d;
        a.groups = (int32_t)groups;
        a.dtype = type_code(xt.scalar_type());
        a.eps = (float)eps;
        a.h = const_cast<void*>(h_ptr);
        a.y = const_cast<void*>(y_ptr);
        a.w_post = static_cast<const float*>(w_post.ptr());
        a.scale = static_cast<const float*>(scale.ptr());
        a.w_pre = static_cast<const float*>(w_pre.ptr());
        if (norm_call(device.index(), &a, c10::cuda::getCurrentCUDAStream(device.index()).stream()) != TTC_OK)
            Py_RETURN_NONE;
        PyObject* first = h_arg.t || changed ? give(args[8], h) : Py_NewRef(args[0]);
        PyObject* second = w_pre.t ? give(args[9], y) : Py_NewRef(Py_None);
        PyObject* both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
        Py_XDECREF(first);
        Py_XDECREF(second);
        return both;
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// (x, h, dy, dh, w_post, z, scale, w_pre, eps, groups, residual): a dict of all gradients
PyObject* norm_grad(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 11 || !norm_grad_call)
        Py_RETURN_NONE;
    try {
        const Arg x(args[0]), h(args[1]), dy(args[2]), dh(args[3]), w_post(args[4]), z(args[5]), scale(args[6]), w_pre(args[7]);
        const double eps = PyFloat_AsDouble(args[8]);
        const long groups = PyErr_Occurred() ? -1 : PyLong_AsLong(args[9]);
        const int residual = PyObject_IsTrue(args[10]);
        if (PyErr_Occurred() || !x.t || residual < 0 || groups < 1 || groups >= INT32_MAX)
            return none();
        const at::Tensor& xt = *x.t;
        if (!xt.is_cuda() || xt.dim() < 1 || type_code(xt.scalar_type()) < 0 || xt.numel() == 0)
            return none();
        const int64_t d = xt.size(xt.dim() - 1);
        const auto device = xt.device();
        ttc_norm_args a = {};
        ttc_norm_grads g = {};
        const void* h_ptr;
        if (d >= INT32_MAX || !dense(w_post, {d}, at::kFloat, device) || !dense(scale, {d}, at::kFloat, device) || !dense(w_pre, {d}, at::kFloat, device) ||
            !flat_rows(x, xt, a.x, a.ldx) || !flat_rows(z, xt, a.z, a.ldz) || !flat_rows(h, xt, h_ptr, a.ldh) || !flat_rows(dy, xt, g.dy, g.lddy) || !flat_rows(dh, xt, g.dh, g.lddh))
            return none();
        a.h = const_cast<void*>(h_ptr);
        a.rows = xt.numel() / d;
        a.d = (int32_t)d;
        a.groups = (int32_t)groups;
        a.dtype = type_code(xt.scalar_type());
        a.eps = (float)eps;
        a.w_post = static_cast<const float*>(w_post.ptr());
        a.scale = static_cast<const float*>(scale.ptr());
        a.w_pre = static_cast<const float*>(w_pre.ptr());
        const auto f32 = xt.options().dtype(at::kFloat);
        at::Tensor dx = at::empty(xt.sizes(), xt.options()), dz, dr, dwp, ds, dw;
        g.dx = dx.data_ptr(), g.lddx = d;
        if (z.t) {
            dz = at::empty(xt.sizes(), xt.options());
            g.dz = dz.data_ptr(), g.lddz = d;
        }
        if (residual) {
            dr = at::empty(xt.sizes(), xt.options());
            g.dresidual = dr.data_ptr(), g.lddr = d;
        }
        auto vector = [&](const Arg& w, at::Tensor& t, float*& to) {
            if (w.t) {
                t = at::empty({d}, f32);
                to = static_cast<float*>(t.data_ptr());
            }
        };
        vector(w_post, dwp, g.dw_post);
        vector(scale, ds, g.dscale);
        vector(w_pre, dw, g.dw_pre);
        const int64_t need = norm_grad_workspace_call(device.index(), &a, &g);
        if (need < 0)
            return none();
        at::Tensor ws;
        if (need > 0)
            ws = at::empty({need}, xt.options().dtype(at::kByte));
        if (norm_grad_call(device.index(), &a, &g, need ? ws.data_ptr() : nullptr, need, c10::cuda::getCurrentCUDAStream(device.index()).stream()) != TTC_OK)
            return none();
        PyObject* o = PyDict_New();
        if (!o || !put(o, "dx", dx) || (z.t && !put(o, "dz", dz)) || (residual && !put(o, "dresidual", dr)) || (w_post.t && !put(o, "dw_post", dwp)) ||
            (scale.t && !put(o, "dscale", ds)) || (w_pre.t && !put(o, "dw_pre", dw))) {
            Py_XDECREF(o);
            return none();
        }
        return o;
    } catch (...) {
        return none();
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

// The same for linear attention and the norms.
PyObject* bind_more(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 12) {
        PyErr_SetString(PyExc_TypeError, "bind_more takes eight addresses and four sizes");
        return nullptr;
    }
    void* at[8];
    for (int i = 0; i < 8; ++i) {
        at[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred())
            return nullptr;
    }
    const long sizes[4] = {(long)sizeof(ttc_decay_args), (long)sizeof(ttc_decay_grads), (long)sizeof(ttc_norm_args), (long)sizeof(ttc_norm_grads)};
    for (int i = 0; i < 4; ++i) {
        const long size = PyLong_AsLong(args[8 + i]);
        if (PyErr_Occurred())
            return nullptr;
        if (size != sizes[i]) {
            PyErr_Format(PyExc_ImportError, "_step.so was built for records of %ld bytes, not %ld: build it again", sizes[i], size);
            return nullptr;
        }
    }
    attention_call = reinterpret_cast<decltype(attention_call)>(at[0]);
    attention_workspace_call = reinterpret_cast<decltype(attention_workspace_call)>(at[1]);
    attention_step_call = reinterpret_cast<decltype(attention_step_call)>(at[2]);
    attention_grad_call = reinterpret_cast<decltype(attention_grad_call)>(at[3]);
    attention_grad_workspace_call = reinterpret_cast<decltype(attention_grad_workspace_call)>(at[4]);
    norm_call = reinterpret_cast<decltype(norm_call)>(at[5]);
    norm_grad_call = reinterpret_cast<decltype(norm_grad_call)>(at[6]);
    norm_grad_workspace_call = reinterpret_cast<decltype(norm_grad_workspace_call)>(at[7]);
    Py_RETURN_NONE;
}

#define TTC_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {TTC_METHOD(bind), TTC_METHOD(conv_step), TTC_METHOD(scan_step), TTC_METHOD(linear), TTC_METHOD(bind_more), TTC_METHOD(attention), TTC_METHOD(attention_grad), TTC_METHOD(norm), TTC_METHOD(norm_grad), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_step", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__step(void) { return PyModule_Create(&module); }
