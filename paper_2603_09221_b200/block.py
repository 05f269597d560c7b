"""Binding of ``include/ttc_block.h``: the operators around the Test-Time Control layer in a block of a language model.

    linear, linear_grad                                            projections with bias, activation and residual
    causal_conv, causal_conv_step, causal_conv_grad                short depthwise causal convolution
    selective_scan, selective_scan_step, selective_scan_grad       state space scan with a diagonal transition

As :mod:`.lqr`, it only marshals arguments: everything runs in the CUDA kernels of ``libttc_lqr.so`` and there is no CPU
fallback.  Calls are enqueued on ``stream`` (a ``torch.cuda.Stream``; default: the current one of the tensors' device) and
do not synchronise; the tensors they are given have to be ready there.  Outputs that are not handed in, and scratch, are
allocated by torch on that stream, so calls may be captured into CUDA graphs.  No autograd graph is recorded: the
gradients are the ``.._grad`` calls.

Token rows are ``[batch, tokens, channels]`` for sequences of equal length, or ``[rows, channels]`` with ``offsets [batch + 1]``
(int32, on the device) for sequences packed one behind the other, or ``[batch, channels]`` in the ``.._step`` calls.  Only
the channels have to be contiguous.
"""
from __future__ import annotations

import ctypes
import os
import struct
import subprocess
import warnings

import torch

from . import build as _build
from . import lqr as _lqr
from .lqr import TTC_BF16, TTC_F32, TtcError, _check, _raw_stream  # noqa: F401

TTC_F16 = 2
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "softplus": 4}

EXPORTS = (
    "ttc_linear", "ttc_linear_workspace", "ttc_linear_grad", "ttc_linear_grad_workspace",
    "ttc_causal_conv", "ttc_causal_conv_step", "ttc_causal_conv_grad", "ttc_causal_conv_grad_workspace",
    "ttc_selective_scan", "ttc_selective_scan_workspace", "ttc_selective_scan_step", "ttc_selective_scan_grad",
    "ttc_selective_scan_grad_workspace", "ttc_block_device_error",
)

_F32 = torch.float32
_DTYPES = {torch.float32: TTC_F32, torch.bfloat16: TTC_BF16, torch.float16: TTC_F16}

# The structures of the header, packed as one record each: filling ctypes fields one by one costs more host time than the
# kernels of a single token take.  ttc_rows is Pqq.
_CONV_ARGS = struct.Struct("qqP4i" + 2 * "Pqq" + "PPPP")
_CONV_GRADS = struct.Struct(2 * "Pqq" + "PPPP")
_SCAN_ARGS = struct.Struct("qqP6i" + 6 * "Pqq" + "PPPPP")
_SCAN_GRADS = struct.Struct(6 * "Pqq" + "PPPPP")
_LINEAR_ARGS = struct.Struct("q6i" + "PPPPPP" + "qqqqq")
_LINEAR_GRADS = struct.Struct("PPPP" + "qqq")
_NO_ROWS = (0, 0, 0)

_lib = None


_step = None                    # the compiled short way into the calls for single tokens, bound to the library when it is loaded


def _load():
    global _lib, _step
    if _lib is None:
        lib = _lqr.load_library()
        p, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        for name in EXPORTS:
            f = getattr(lib, name)
            f.restype = ctypes.c_int
            grads = [p] if "_grad" in name else []
            if name == "ttc_block_device_error":
                f.argtypes = [i32, ctypes.POINTER(ctypes.c_int32)]
            elif name.endswith("_workspace"):
                f.restype = i64
                f.argtypes = [i32, p] + grads
            elif name in ("ttc_causal_conv", "ttc_causal_conv_step", "ttc_selective_scan_step"):
                f.argtypes = [i32, p, p]
            else:
                f.argtypes = [i32, p] + grads + [p, i64, p]
        _lib, _step = lib, _short_way(lib)
    return _lib


class _LongWay:
    """Stands in for the compiled module where it cannot be built: every call is marshalled here."""
    conv_step = scan_step = linear = staticmethod(lambda *args: None)


def _short_way(lib):
    try:
        if not os.path.exists(_build.STEP) or os.environ.get("TTC_LQR_REBUILD"):
            _build.build_step_binding(force=True)
        from . import _step as step
        # with the records' sizes: one that was compiled with another header is refused
        step.bind(*(ctypes.cast(getattr(lib, k), ctypes.c_void_p).value
                    for k in ("ttc_causal_conv_step", "ttc_selective_scan_step", "ttc_linear", "ttc_linear_workspace")),
                  _CONV_ARGS.size, _SCAN_ARGS.size, _LINEAR_ARGS.size)
    except (ImportError, OSError, TypeError, subprocess.CalledProcessError) as e:
        warnings.warn("single-token calls take the slower way through Python: %s" % e)
        return _LongWay
    return step


def _type_of(t, f32=True):
    code = _DTYPES.get(t.dtype)
    if code is None or (code == TTC_F32 and not f32):
        raise TypeError("x must be %sbfloat16 or float16, got %s" % ("float32, " if f32 else "", t.dtype))
    return code


def _explain(t, name, shape, dtype, device):
    """Raises for a tensor that did not pass one of the checks below."""
    shape = tuple(shape)
    if t.get_device() != device:
        raise ValueError("%s is on %s, x on device %d" % (name, t.device, device))
    if tuple(t.shape) != shape or t.dtype != dtype:
        raise ValueError("%s must have shape %s and type %s, got %s, %s" % (name, shape, dtype, tuple(t.shape), t.dtype))
    raise ValueError("%s must be contiguous (token rows: in their channels), got strides %s" % (name, t.stride()))


def _dense(t, name, shape, device, dtype=_F32):
    """Address of a contiguous tensor of that shape and type (0: missing)."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        _explain(t, name, shape, dtype, device)
    return t.data_ptr()


def _rows3(t, name, shape, device, dtype):
    """``(ptr, bstride, tstride)`` of ``[batch, tokens, channels]``."""
    if t is None:
        return _NO_ROWS
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _explain(t, name, shape, dtype, device)
    b, s, c = t.stride()
    if c != 1 and shape[2] > 1:
        _explain(t, name, shape, dtype, device)
    return t.data_ptr(), b, s


def _rows2(t, name, shape, device, dtype):
    """``(ptr, 0, tstride)`` of ``[rows, channels]``."""
    if t is None:
        return _NO_ROWS
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _explain(t, name, shape, dtype, device)
    s, c = t.stride()
    if c != 1 and shape[1] > 1:
        _explain(t, name, shape, dtype, device)
    return t.data_ptr(), 0, s


def _rows1(t, name, shape, device, dtype):
    """``(ptr, bstride, 0)`` of ``[batch, channels]``: one token of each sequence."""
    if t is None:
        return _NO_ROWS
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _explain(t, name, shape, dtype, device)
    s, c = t.stride()
    if c != 1 and shape[1] > 1:
        _explain(t, name, shape, dtype, device)
    return t.data_ptr(), s, 0


def _shared(t, name, lead, device, dtype, n, groups, rows):
    """Rows of B or C, ``[*lead, n]`` or ``[*lead, groups, n]``."""
    if t is None:
        return _NO_ROWS
    shape, stride, k = t.shape, t.stride(), len(lead)
    if len(shape) == k + 1:
        if groups != 1 or shape[k] != n or (n > 1 and stride[k] != 1):
            _explain(t, name, (*lead, groups, n) if groups > 1 else (*lead, n), dtype, device)
    elif len(shape) != k + 2 or shape[k] != groups or shape[k + 1] != n or (n > 1 and stride[k + 1] != 1) or (groups > 1 and stride[k] != n):
        _explain(t, name, (*lead, groups, n), dtype, device)
    if shape[:k] != lead or t.dtype is not dtype or t.get_device() != device:
        _explain(t, name, (*lead, *shape[k:]), dtype, device)
    if k == 2:
        return t.data_ptr(), stride[0], stride[1]
    return (t.data_ptr(), stride[0], 0) if rows is _rows1 else (t.data_ptr(), 0, stride[0])


def _sequences(x, offsets):
    """Number of sequences, tokens (of each, or of all), address of the offsets, and the form of the rows."""
    shape = x.shape
    if offsets is None:
        if len(shape) != 3:
            raise ValueError("x must be [batch, tokens, channels] (or [rows, channels] with offsets)")
        return shape[0], shape[1], 0, _rows3
    if len(shape) != 2:
        raise ValueError("x must be [rows, channels] with offsets")
    if offsets.dim() != 1 or offsets.shape[0] < 1 or offsets.dtype != torch.int32 or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous int32 tensor [batch + 1]")
    if offsets.get_device() != x.get_device():
        raise ValueError("offsets is on %s, x on %s" % (offsets.device, x.device))
    return offsets.shape[0] - 1, shape[0], offsets.data_ptr(), _rows2


def _device_of(x):
    """Checked behind the shapes, so that those are refused without a GPU too."""
    index = x.get_device()
    if index < 0:
        raise ValueError("the operators run on CUDA tensors only, got %s" % x.device)
    return index


def _raw(index, stream):
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(index) if _raw_stream else torch.cuda.current_stream(index).cuda_stream


def _like(x, stream):
    if stream is None:
        return torch.empty_like(x)
    with torch.cuda.stream(stream):
        return torch.empty_like(x)


def _empty(shape, dtype, x, stream):
    if stream is None:
        return x.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return x.new_empty(shape, dtype=dtype)


def _workspace(need, x, stream):
    """Scratch of that many bytes (a status where negative), and its address."""
    if need <= 0:
        _check(need)
        return None, 0
    ws = _empty((need,), torch.uint8, x, stream)
    return ws, ws.data_ptr()


def _outputs(want, out, shapes, x, stream):
    got = {}
    for k in want:
        t = None if out is None else out.get(k)
        got[k] = t if t is not None else _empty(*shapes[k], x, stream)
    return got


# ---- causal convolution -------------------------------------------------------------------------------------------------

def _conv_taps(x, w, act):
    code = _type_of(x)
    a = ACTIVATIONS.get(act)
    if a is None:
        raise ValueError("unknown activation %r" % (act,))
    d = x.shape[-1]
    if w.dim() != 2 or w.shape[0] != d:
        raise ValueError("w must be [channels, taps]")
    return code, a, d, w.shape[1]


def _conv_record(x, w, bias, act, state, offsets, y, state_out):
    batch, tokens, off, rows = _sequences(x, offsets)
    code, a, d, taps = _conv_taps(x, w, act)
    dev, dtype, shape, window = x.get_device(), x.dtype, x.shape, (batch, taps - 1, d)
    return _CONV_ARGS.pack(batch, tokens, off, d, taps, a, code, *rows(x, "x", shape, dev, dtype), *rows(y, "y", shape, dev, dtype),
                           _dense(w, "w", (d, taps), dev), _dense(bias, "bias", (d,), dev), _dense(state, "state", window, dev, dtype),
                           _dense(state_out, "state_out", window, dev, dtype)), window, rows


def causal_conv(x, w, bias=None, act="none", state=None, offsets=None, y=None, state_out=None, stream=None):
    """``y_t = act(bias + sum_j w[:, j] x_{t - (taps - 1) + j})`` per channel (``ttc_causal_conv``).

    ``w [channels, taps]`` (2 to 4 taps) and ``bias [channels]`` float32; ``state [batch, taps - 1, channels]`` holds the inputs
    in front of the sequences (default: zeros), ``state_out`` receives the last ones and may be ``state``.  Returns ``y``."""
    if y is None:
        y = _like(x, stream)
    record, _, _ = _conv_record(x, w, bias, act, state, offsets, y, state_out)
    index = _device_of(x)
    status = _load().ttc_causal_conv(index, record, _raw(index, stream))
    if status:
        _check(status)
    return y


def causal_conv_step(x, w, state, bias=None, act="none", y=None, stream=None):
    """One token of each sequence, ``x [batch, channels]``: as :func:`causal_conv`; ``state`` moves on in place."""
    if stream is None:
        if _step is None:
            _load()
        got = _step.conv_step(x, w, state, bias, ACTIVATIONS.get(act, -1), y)
        if got is not None:
            return got
    if y is None:
        y = _like(x, stream)
    if x.dim() != 2:
        raise ValueError("x must be [batch, channels]")
    code, a, d, taps = _conv_taps(x, w, act)
    dev, dtype, shape = x.get_device(), x.dtype, x.shape
    record = _CONV_ARGS.pack(shape[0], 1, 0, d, taps, a, code, *_rows1(x, "x", shape, dev, dtype), *_rows1(y, "y", shape, dev, dtype),
                             _dense(w, "w", (d, taps), dev), _dense(bias, "bias", (d,), dev), 0,
                             _dense(state, "state", (shape[0], taps - 1, d), dev, dtype))
    if dev < 0:
        _device_of(x)
    status = (_lib or _load()).ttc_causal_conv_step(dev, record, _raw(dev, stream))
    if status:
        _check(status)
    return y


CONV_GRAD_KEYS = ("dx", "dw", "dbias", "dstate")


def causal_conv_grad(dy, x, w, bias=None, act="none", state=None, offsets=None, dstate_out=None, want=CONV_GRAD_KEYS, out=None,
                     stream=None):
    """Gradients of :func:`causal_conv` given ``dy`` and that of ``state_out`` (``dstate_out``; default: zero).  Returns a dict
    with the wanted of ``dx, dw, dbias, dstate``; ``out`` may hold tensors to write them to."""
    record, window, rows = _conv_record(x, w, bias, act, state, offsets, None, None)
    index = _device_of(x)
    shape, dtype = x.shape, x.dtype
    shapes = {"dx": (shape, dtype), "dw": (w.shape, _F32), "dbias": (shape[-1:], _F32), "dstate": (window, dtype)}
    got = _outputs(want, out, shapes, x, stream)
    grads = _CONV_GRADS.pack(*rows(dy, "dy", shape, index, dtype), *rows(got.get("dx"), "dx", shape, index, dtype),
                             _dense(dstate_out, "dstate_out", window, index, dtype), _dense(got.get("dw"), "dw", w.shape, index),
                             _dense(got.get("dbias"), "dbias", shape[-1:], index), _dense(got.get("dstate"), "dstate", window, index, dtype))
    lib = _load()
    need = lib.ttc_causal_conv_grad_workspace(index, record, grads)
    ws, at = _workspace(need, x, stream)
    _check(lib.ttc_causal_conv_grad(index, record, grads, at, need, _raw(index, stream)))
    return got


# ---- selective scan -----------------------------------------------------------------------------------------------------

def _states(A, B, lead):
    """Number of states and of groups."""
    extra = B.dim() - lead
    if extra not in (1, 2):
        raise ValueError("B must be [.., n] or [.., groups, n]")
    if A.dim() != 2:
        raise ValueError("A must be [channels, n]")
    return B.shape[-1], 1 if extra == 1 else B.shape[-2]


def _scan_record(x, delta, A, B, C, D, z, delta_bias, softplus, state, offsets, y, state_out):
    batch, tokens, off, rows = _sequences(x, offsets)
    code, shape, t, dev = _type_of(x), x.shape, x.dtype, x.get_device()
    lead, d = tuple(shape[:-1]), shape[-1]
    n, groups = _states(A, B, len(lead))
    states = (batch, d, n)
    return _SCAN_ARGS.pack(batch, tokens, off, d, n, groups, code, 1 if softplus else 0, 0,
                           *rows(x, "x", shape, dev, t), *rows(delta, "delta", shape, dev, t),
                           *_shared(B, "B", lead, dev, t, n, groups, rows), *_shared(C, "C", lead, dev, t, n, groups, rows),
                           *rows(z, "z", shape, dev, t), *rows(y, "y", shape, dev, t),
                           _dense(A, "A", (d, n), dev), _dense(D, "D", (d,), dev), _dense(delta_bias, "delta_bias", (d,), dev),
                           _dense(state, "state", states, dev), _dense(state_out, "state_out", states, dev)), states, rows, n, groups


def selective_scan(x, delta, A, B, C, D=None, z=None, delta_bias=None, softplus=False, state=None, offsets=None, y=None,
                   state_out=None, stream=None):
    """``h_t = exp(D_t A) h_{t-1} + D_t x_t B_t``, ``y_t = (C_t . h_t + D x_t) silu(z_t)`` (``ttc_selective_scan``), where
    ``D_t = delta_t + delta_bias``, or its softplus.

    ``x, delta, z`` are rows of channels, ``B, C`` rows ``[.., n]`` or ``[.., groups, n]`` (1 to 128 states); ``A [channels, n]``,
    ``D, delta_bias [channels]`` and ``state, state_out [batch, channels, n]`` float32.  ``state`` is h in front of the sequences
    (default: zero), ``state_out`` receives the last ones and may be ``state``.  Returns ``y``."""
    if y is None:
        y = _like(x, stream)
    record = _scan_record(x, delta, A, B, C, D, z, delta_bias, softplus, state, offsets, y, state_out)[0]
    index = _device_of(x)
    lib = _load()
    need = lib.ttc_selective_scan_workspace(index, record)
    ws, at = _workspace(need, x, stream)
    status = lib.ttc_selective_scan(index, record, at, need, _raw(index, stream))
    if status:
        _check(status)
    return y


def selective_scan_step(x, delta, A, B, C, state, D=None, z=None, delta_bias=None, softplus=False, y=None, stream=None):
    """One token of each sequence, ``x [batch, channels]``: as :func:`selective_scan`; ``state`` moves on in place."""
    if stream is None:
        if _step is None:
            _load()
        got = _step.scan_step(x, delta, A, B, C, state, D, z, delta_bias, softplus, y)
        if got is not None:
            return got
    if y is None:
        y = _like(x, stream)
    if x.dim() != 2:
        raise ValueError("x must be [batch, channels]")
    code, shape, t, dev = _type_of(x), x.shape, x.dtype, x.get_device()
    batch, d = shape
    n, groups = _states(A, B, 1)
    record = _SCAN_ARGS.pack(batch, 1, 0, d, n, groups, code, 1 if softplus else 0, 0,
                             *_rows1(x, "x", shape, dev, t), *_rows1(delta, "delta", shape, dev, t),
                             *_shared(B, "B", (batch,), dev, t, n, groups, _rows1), *_shared(C, "C", (batch,), dev, t, n, groups, _rows1),
                             *_rows1(z, "z", shape, dev, t), *_rows1(y, "y", shape, dev, t),
                             _dense(A, "A", (d, n), dev), _dense(D, "D", (d,), dev), _dense(delta_bias, "delta_bias", (d,), dev),
                             0, _dense(state, "state", (batch, d, n), dev))
    if dev < 0:
        _device_of(x)
    status = (_lib or _load()).ttc_selective_scan_step(dev, record, _raw(dev, stream))
    if status:
        _check(status)
    return y


SCAN_GRAD_KEYS = ("dx", "ddelta", "dz", "dB", "dC", "dA", "dD", "ddelta_bias", "dstate")


def selective_scan_grad(dy, x, delta, A, B, C, D=None, z=None, delta_bias=None, softplus=False, state=None, offsets=None,
                        dstate_out=None, want=None, out=None, stream=None):
    """Gradients of :func:`selective_scan` given ``dy`` and that of ``state_out`` (``dstate_out``; default: zero).  Returns a
    dict with the wanted of ``dx, ddelta, dz, dB, dC, dA, dD, ddelta_bias, dstate`` (default: all, without ``dz`` where there
    is no ``z``); ``out`` may hold tensors to write them to."""
    record, states, rows, n, groups = _scan_record(x, delta, A, B, C, D, z, delta_bias, softplus, state, offsets, None, None)
    index = _device_of(x)
    shape, t = x.shape, x.dtype
    lead, d = tuple(shape[:-1]), shape[-1]
    if want is None:
        want = SCAN_GRAD_KEYS if z is not None else [k for k in SCAN_GRAD_KEYS if k != "dz"]
    shapes = {"dx": (shape, t), "ddelta": (shape, t), "dz": (shape, t), "dB": (B.shape, t), "dC": (C.shape, t), "dA": (A.shape, _F32),
              "dD": ((d,), _F32), "ddelta_bias": ((d,), _F32), "dstate": (states, _F32)}
    got = _outputs(want, out, shapes, x, stream)
    grads = _SCAN_GRADS.pack(*rows(dy, "dy", shape, index, t), *rows(got.get("dx"), "dx", shape, index, t),
                             *rows(got.get("ddelta"), "ddelta", shape, index, t),
                             *_shared(got.get("dB"), "dB", lead, index, t, n, groups, rows),
                             *_shared(got.get("dC"), "dC", lead, index, t, n, groups, rows),
                             *rows(got.get("dz"), "dz", shape, index, t), _dense(dstate_out, "dstate_out", states, index),
                             _dense(got.get("dA"), "dA", A.shape, index), _dense(got.get("dD"), "dD", (d,), index),
                             _dense(got.get("ddelta_bias"), "ddelta_bias", (d,), index), _dense(got.get("dstate"), "dstate", states, index))
    lib = _load()
    need = lib.ttc_selective_scan_grad_workspace(index, record, grads)
    ws, at = _workspace(need, x, stream)
    _check(lib.ttc_selective_scan_grad(index, record, grads, at, need, _raw(index, stream)))
    return got


# ---- projections --------------------------------------------------------------------------------------------------------

def _on(stream, f):
    """f() with `stream` as the current one."""
    if stream is None:
        return f()
    with torch.cuda.stream(stream):
        return f()


def _matrix(t, name, cols, dtype, device, rows=None, stream=None, output=False):
    """``t`` as ``[rows, cols]``, its address, rows and row stride.  Leading dimensions are taken together; inputs whose rows
    no single stride describes, or lie over one another (a row for all tokens, by ``expand``), are copied."""
    if t is None:
        return None, 0, 0, 0
    shape = t.shape
    if len(shape) < 1 or shape[-1] != cols or t.dtype is not dtype or t.get_device() != device:
        _explain(t, name, (*shape[:-1], cols), dtype, device)
    if len(shape) != 2:
        lead = (-1, cols) if t.numel() else (0, cols)
        t = t.view(lead) if output else _on(stream, lambda: t.reshape(lead))
        shape = t.shape
    ld, one = t.stride()
    if (one != 1 and cols > 1 and shape[0]) or (rows is not None and shape[0] != rows):
        raise ValueError("%s must be %s rows of contiguous elements, got %s with strides %s" % (name, rows, tuple(shape), t.stride()))
    if ld < cols and shape[0] > 1 and not output:
        t, ld = _on(stream, t.contiguous), cols
    return t, t.data_ptr(), shape[0], ld


def linear(x, w, bias=None, act="none", residual=None, y=None, pre=None, out_dtype=None, stream=None):
    """``act(x W' + bias) + residual`` (``ttc_linear``).

    ``x [.., k]`` and ``w [m, k]`` bfloat16 or float16; ``bias [m]`` float32; ``residual`` and the result ``[.., m]`` have
    ``out_dtype``: the type of ``x`` (default; that of ``y`` where it is given), or float32.  ``act`` is one of ``ACTIVATIONS``.  ``pre``
    receives what the activation was given, in the type of ``x``; :func:`linear_grad` wants it.  Returns ``y``, which may be ``residual``."""
    dtype, dev = x.dtype, x.get_device()
    if out_dtype is None:
        out_dtype = y.dtype if y is not None else dtype
    if stream is None and pre is None and (out_dtype is dtype or out_dtype is _F32):
        if _step is None:
            _load()
        got = _step.linear(x, w, bias, ACTIVATIONS.get(act, -1), residual, y, out_dtype is _F32)
        if got is not None:
            return got
    code, a = _type_of(x, False), ACTIVATIONS.get(act)
    if a is None:
        raise ValueError("unknown activation %r" % (act,))
    if w.dim() != 2:
        raise ValueError("w must be [m, k]")
    if out_dtype is not dtype and out_dtype is not _F32:
        raise TypeError("outputs are of x's type or float32, not %s" % out_dtype)
    m, k = w.shape
    x2, px, rows, ldx = _matrix(x, "x", k, dtype, dev, None, stream)
    w2, pw, _, ldw = _matrix(w, "w", k, dtype, dev, None, stream)
    if residual is not None and residual.shape[:-1] != x.shape[:-1]:
        raise ValueError("residual must be %s, got %s" % ((*x.shape[:-1], m), tuple(residual.shape)))
    r2, pr, _, ldr = _matrix(residual, "residual", m, out_dtype, dev, rows, stream)
    _, pp, _, ldp = _matrix(pre, "pre", m, dtype, dev, rows, None, True)
    pb = _dense(bias, "bias", (m,), dev)
    if dev < 0:
        _device_of(x)
    if y is None:
        y = _empty((*x.shape[:-1], m), out_dtype, x, stream)
    _, py, _, ldy = _matrix(y, "y", m, out_dtype, dev, rows, None, True)
    record = _LINEAR_ARGS.pack(rows, k, m, code, _DTYPES[out_dtype], a, 0, px, pw, pb, pr, py, pp, ldx, ldw, ldr, ldy, ldp)
    lib = _lib or _load()
    need = lib.ttc_linear_workspace(dev, record)
    ws, at = _workspace(need, x, stream) if need else (None, 0)
    status = lib.ttc_linear(dev, record, at, need, _raw(dev, stream))
    if status:
        _check(status)
    return y


LINEAR_GRAD_KEYS = ("dx", "dw", "dbias")


def linear_grad(dy, x, w, act="none", pre=None, want=LINEAR_GRAD_KEYS, out=None, stream=None):
    """Gradients of :func:`linear` given ``dy`` (the residual's gradient is ``dy`` itself); ``pre`` as the forward call wrote it
    (needed unless ``act`` is ``"none"``).  Returns a dict with the wanted of ``dx`` and ``dw`` (type of ``x``) and ``dbias``
    (float32); ``out`` may hold tensors to write them to."""
    dtype, dev = x.dtype, x.get_device()
    code, a = _type_of(x, False), ACTIVATIONS.get(act)
    if a is None:
        raise ValueError("unknown activation %r" % (act,))
    if w.dim() != 2:
        raise ValueError("w must be [m, k]")
    m, k = w.shape
    if dy.dtype is not dtype and dy.dtype is not _F32:
        raise TypeError("dy is of x's type or float32, not %s" % dy.dtype)
    if dy.shape != (*x.shape[:-1], m):
        raise ValueError("dy must be %s, got %s" % ((*x.shape[:-1], m), tuple(dy.shape)))
    x2, px, rows, ldx = _matrix(x, "x", k, dtype, dev, None, stream)
    w2, pw, _, ldw = _matrix(w, "w", k, dtype, dev, None, stream)
    p2, pp, _, ldp = _matrix(pre, "pre", m, dtype, dev, rows, stream)
    d2, pdy, _, lddy = _matrix(dy, "dy", m, dy.dtype, dev, rows, stream)
    _device_of(x)
    shapes = {"dx": (x.shape, dtype), "dw": (w.shape, dtype), "dbias": ((m,), _F32)}
    got = _outputs(want, out, shapes, x, stream)
    _, pdx, _, lddx = _matrix(got.get("dx"), "dx", k, dtype, dev, rows, None, True)
    _, pdw, _, lddw = _matrix(got.get("dw"), "dw", k, dtype, dev, m, None, True)
    record = _LINEAR_ARGS.pack(rows, k, m, code, _DTYPES[dy.dtype], a, 0, px, pw, 0, 0, 0, pp, ldx, ldw, 0, 0, ldp)
    grads = _LINEAR_GRADS.pack(pdy, pdx, pdw, _dense(got.get("dbias"), "dbias", (m,), dev), lddy, lddx, lddw)
    lib = _load()
    need = lib.ttc_linear_grad_workspace(dev, record, grads)
    ws, at = _workspace(need, x, stream)
    _check(lib.ttc_linear_grad(dev, record, grads, at, need, _raw(dev, stream)))
    return got


def device_error(device=0):
    """``ttc_block_device_error``: whether a bounded wait of the matrix products has given up on the device."""
    value = ctypes.c_int32(-1)
    _check(_load().ttc_block_device_error(int(device), ctypes.byref(value)))
    return value.value
