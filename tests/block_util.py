"""Plain 64-bit forms of the operators of include/ttc_block.h, with the bounds that tests hold the kernels to.

Bounds.  u = 2^-24 is half a step of float32.  A result is a sum of products; every product passes a number of float32
operations, each with a relative error of at most u (2^-22 for ex2.approx, an argument t = D_t A log2(e) with a few u of
relative error moves exp by |t| times that).  So |error| <= R u S to first order, where S is the same sum taken over the
products' magnitudes and R the longest path's count; what is rounded to 16 bits adds half a step of the result.  S comes out
of the same code run on magnitudes (`magnitudes=True`).
"""
import numpy as np
import torch

U = 2.0 ** -24


def half_step(dtype):
    return 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy()


def within(got, want, bound, dtype, what=""):
    """got (tensor) against want and an absolute bound on its float32 error (arrays); the rounding to `dtype` comes on top."""
    assert got.dtype == dtype and tuple(got.shape) == tuple(want.shape), (what, got.shape, want.shape)
    g = f64(got)
    finite = np.isfinite(want)
    assert np.array_equal(np.isnan(g), np.isnan(want)), what
    assert np.array_equal(g[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)]), what
    tiny = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126                 # half a step of the smallest numbers
    room = bound * (1 + half_step(dtype)) + half_step(dtype) * np.abs(want) + tiny
    off = np.abs(g - want)[finite] - np.broadcast_to(room, want.shape)[finite]
    assert off.size == 0 or off.max() <= 0, "%s: %g over the bound (%g), values up to %g" % (
        what, off.max(), np.broadcast_to(room, want.shape)[finite][off.argmax()], np.abs(want[finite]).max())


def sigmoid(z):
    return 0.5 * (1 + np.tanh(0.5 * z))


def silu(z):
    return z * sigmoid(z)


def silu_slope(z):
    p = sigmoid(z)
    return p * (1 + z * (1 - p))


def spans(lead, offsets):
    if offsets is not None:
        o = [int(v) for v in offsets]
        return [(o[i], o[i + 1]) for i in range(len(o) - 1)]
    batch, tokens = lead
    return [(b * tokens, (b + 1) * tokens) for b in range(batch)]


# ---- causal convolution --------------------------------------------------------------------------------------------------

def conv(x, w, bias, act, state, seqs):
    """x [rows, d], state [batch, taps - 1, d] or None; returns y, the last windows, z."""
    taps = w.shape[1]
    y, z = np.full_like(x, np.nan), np.full_like(x, np.nan)
    last = np.zeros((len(seqs), taps - 1, x.shape[1]))
    for b, (lo, hi) in enumerate(seqs):
        front = state[b] if state is not None else np.zeros((taps - 1, x.shape[1]))
        line = np.concatenate([front, x[lo:hi]])
        for t in range(hi - lo):
            z[lo + t] = (line[t:t + taps] * w.T).sum(0) + (0 if bias is None else bias)
        last[b] = line[hi - lo:]
    y = silu(z) if act == "silu" else z
    return y, last, z


def conv_grad(dy, x, w, bias, act, state, seqs, dlast, magnitudes=False):
    taps, d = w.shape[1], x.shape[1]
    _, _, z = conv(x, w, bias, act, state, seqs)
    slope = silu_slope(z) if act == "silu" else np.ones_like(z)
    m = np.abs if magnitudes else (lambda v: v)
    dy, x, w, slope = m(dy), m(x), m(w), m(slope)
    state = None if state is None else m(state)
    dx, dw, db = np.full_like(x, np.nan), np.zeros_like(w), np.zeros(d)
    dstate = np.zeros((len(seqs), taps - 1, d))
    for b, (lo, hi) in enumerate(seqs):
        front = state[b] if state is not None else np.zeros((taps - 1, d))
        line, dline = np.concatenate([front, x[lo:hi]]), np.zeros((taps - 1 + hi - lo, d))
        if dlast is not None:
            dline[hi - lo:] += m(dlast[b])
        for t in range(hi - lo):
            dz = dy[lo + t] * slope[lo + t]
            dw += (line[t:t + taps] * dz).T
            db += dz
            dline[t:t + taps] += dz * w.T
        dstate[b], dx[lo:hi] = dline[:taps - 1], dline[taps - 1:]
    return {"dx": dx, "dw": dw, "dbias": db, "dstate": dstate}


# ---- selective scan ------------------------------------------------------------------------------------------------------

def scan_step_sizes(delta, delta_bias, softplus):
    raw = delta + (0 if delta_bias is None else delta_bias)
    return (np.logaddexp(raw, 0), sigmoid(raw)) if softplus else (raw, np.ones_like(raw))


def scan(x, delta, A, B, C, D, z, delta_bias, softplus, state, seqs, magnitudes=False):
    """x, delta, z [rows, d], B, C [rows, groups, n], state [batch, d, n] or None; returns y, the last states, all states."""
    rows, d = x.shape
    step, _ = scan_step_sizes(delta, delta_bias, softplus)
    m = np.abs if magnitudes else (lambda v: v)
    gate = m(silu(z)) if z is not None else np.ones_like(x)
    share = d // B.shape[1]
    wide = lambda v: np.repeat(m(v), share, 0)  # noqa: E731
    y, hs = np.full_like(x, np.nan), np.full((rows, d, A.shape[1]), np.nan)
    last = np.zeros((len(seqs), d, A.shape[1]))
    for b, (lo, hi) in enumerate(seqs):
        h = m(state[b]).copy() if state is not None else np.zeros((d, A.shape[1]))
        for t in range(lo, hi):
            h = np.exp(step[t][:, None] * A) * h + m(step[t] * x[t])[:, None] * wide(B[t])
            hs[t] = h
            y[t] = ((h * wide(C[t])).sum(1) + (0 if D is None else m(D) * m(x[t]))) * gate[t]
        last[b] = h
    return y, last, hs


def scan_grad(dy, x, delta, A, B, C, D, z, delta_bias, softplus, state, seqs, dlast, magnitudes=False):
    rows, d = x.shape
    n, groups = A.shape[1], B.shape[1]
    step, chain = scan_step_sizes(delta, delta_bias, softplus)
    _, _, hs = scan(x, delta, A, B, C, D, z, delta_bias, softplus, state, seqs, magnitudes)
    m = np.abs if magnitudes else (lambda v: v)
    gate = m(silu(z)) if z is not None else np.ones_like(x)
    share = d // groups
    wide = lambda v: np.repeat(m(v), share, 0)  # noqa: E731
    narrow = lambda v: v.reshape(groups, share, n).sum(1)  # noqa: E731
    skip = np.zeros(d) if D is None else m(D)
    out = {k: np.full_like(x, np.nan) for k in ("dx", "ddelta", "dz")}
    out.update(dB=np.full_like(B, np.nan), dC=np.full_like(C, np.nan), dA=np.zeros_like(A), dD=np.zeros(d), ddelta_bias=np.zeros(d),
               dstate=np.zeros((len(seqs), d, n)))
    for b, (lo, hi) in enumerate(seqs):
        q = m(dlast[b]).copy() if dlast is not None else np.zeros((d, n))
        for t in range(hi - 1, lo - 1, -1):
            g = m(dy[t]) * gate[t]
            before = hs[t - 1] if t > lo else (m(state[b]) if state is not None else np.zeros((d, n)))
            a = np.exp(step[t][:, None] * A)
            q = q + wide(C[t]) * g[:, None]
            out["dC"][t] = narrow(hs[t] * g[:, None])
            out["dB"][t] = narrow(q * m(step[t] * x[t])[:, None])
            qB = (q * wide(B[t])).sum(1)
            through = q * a * before
            out["dx"][t] = m(step[t]) * qB + skip * g
            ds = (m(x[t]) * qB + (through * m(A)).sum(1)) * chain[t]
            out["ddelta"][t] = ds
            out["ddelta_bias"] += ds
            out["dA"] += through * m(step[t])[:, None]
            out["dD"] += g * m(x[t])
            if z is not None:
                out["dz"][t] = m(dy[t]) * ((hs[t] * wide(C[t])).sum(1) + skip * m(x[t])) * m(silu_slope(z[t]))
            q = a * q
        out["dstate"][b] = q
    if z is None:
        del out["dz"]
    return out


def scan_roundings(longest, rows, d, n, largest):
    """R of the bounds above for a scan: per token of the longest sequence one exponential (2^-22 = 4 u, and an argument with at
    most 6 u of relative error from the step size, A log2(e) and their product), its product and a sum; the sums over states,
    channels and rows; two dozen more for the step size, the gates and the products of an output."""
    return longest * (6 + 6 * largest) + n + d + rows + 24
