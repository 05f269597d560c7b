"""Plain 64-bit forms of linear attention with a decay for each head and of the norms around a block, token by token and row by row, with
the bounds that tests hold the kernels to.

Bounds.  u = 2^-24 and h are half a step of float32 and of the rows' type.  Results are sums of products; S is the same sum over the
products' magnitudes (`magnitudes=True`).  Each product passes float32 operations: a contraction over dk, dv or 128 tokens, each of whose
additions in the tensor cores may cut off two u of the partial sum; exponentials (4 u, and 8 u of an argument of size L, the sum of log2 decays over a
chunk); two more for each chunk that a state is carried over.  Scores, and the state that queries (of the gradients of v: keys) meet, are
rounded to the rows' type once: h.  So |error| <= (h + R u) S for rows, and R u S for what is float32.
"""
import numpy as np

from tests.block_util import U, f64, half_step, scan_step_sizes, sigmoid, silu, silu_slope, spans, within  # noqa: F401

CHUNK = 128


def step_sizes(delta, delta_bias, softplus, rows, heads):
    if delta is None:
        return np.ones((rows, heads)), np.zeros((rows, heads))
    with np.errstate(invalid="ignore"):
        return scan_step_sizes(delta, delta_bias, softplus)


def attend(q, k, v, A, delta, delta_bias, softplus, scale, state, seqs, magnitudes=False):
    """q, k [rows, groups, dk], v [rows, heads, dv], state [batch, heads, dk, dv] or None; returns y, the last states, the states
    in front of every row, the decays."""
    rows, heads, dv = v.shape
    m = np.abs if magnitudes else (lambda x: x)
    share = heads // q.shape[1]
    q, k, v = (np.repeat(m(q), share, 1) * abs(scale) if magnitudes else np.repeat(q, share, 1) * scale), np.repeat(m(k), share, 1), m(v)
    step, _ = step_sizes(delta, delta_bias, softplus, rows, heads)
    a = np.exp(A * step)
    y, before = np.full_like(v, np.nan), np.zeros((rows, heads, q.shape[2], dv))
    last = np.zeros((len(seqs), heads, q.shape[2], dv))
    for b, (lo, hi) in enumerate(seqs):
        S = m(state[b]).copy() if state is not None else np.zeros_like(last[0])
        for t in range(lo, hi):
            before[t] = S
            S = a[t][:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
            y[t] = np.einsum("hk,hkv->hv", q[t], S)
        last[b] = S
    return y, last, before, a


def attend_grad(dy, q, k, v, A, delta, delta_bias, softplus, scale, state, seqs, dlast, magnitudes=False):
    rows, heads, dv = v.shape
    groups, dk = q.shape[1:]
    share = heads // groups
    m = np.abs if magnitudes else (lambda x: x)
    _, _, before, a = attend(q, k, v, A, delta, delta_bias, softplus, scale, state, seqs, magnitudes)
    s = abs(scale) if magnitudes else scale
    wq, wk, v, dy = np.repeat(m(q), share, 1), np.repeat(m(k), share, 1), m(v), m(dy)
    step, slope = step_sizes(delta, delta_bias, softplus, rows, heads)
    out = {"dq": np.full((rows, heads, dk), np.nan), "dk": np.full((rows, heads, dk), np.nan), "dv": np.full_like(v, np.nan),
           "ddelta": np.full((rows, heads), np.nan), "dA": np.zeros(heads), "ddelta_bias": np.zeros(heads),
           "dstate": np.zeros((len(seqs), heads, dk, dv))}
    for b, (lo, hi) in enumerate(seqs):
        Z = m(dlast[b]).copy() if dlast is not None else np.zeros((heads, dk, dv))
        for t in range(hi - 1, lo - 1, -1):
            S = a[t][:, None, None] * before[t] + wk[t][:, :, None] * v[t][:, None, :]
            out["dq"][t] = s * np.einsum("hkv,hv->hk", S, dy[t])
            Z = Z + s * wq[t][:, :, None] * dy[t][:, None, :]
            out["dk"][t] = np.einsum("hkv,hv->hk", Z, v[t])
            out["dv"][t] = np.einsum("hkv,hk->hv", Z, wk[t])
            Z = a[t][:, None, None] * Z
            dl = (Z * before[t]).sum((1, 2))
            out["dA"] += dl * m(step[t])
            out["ddelta"][t] = dl * m(A) * m(slope[t])
            out["ddelta_bias"] += out["ddelta"][t]
        out["dstate"][b] = Z
    for n in ("dq", "dk"):
        out[n] = out[n].reshape(rows, groups, share, dk).sum(2)
    if delta is None:
        del out["ddelta"], out["ddelta_bias"]
    return out


def roundings(dk, dv, longest, A, delta, delta_bias, softplus, rows, heads):
    """R of the bounds above, for outputs and states; gradients pass twice as much, their sums over the tokens (in shares of a chunk, then chunk by chunk) 256 and
    the chunks more."""
    step, _ = step_sizes(delta, delta_bias, softplus, rows, heads)
    with np.errstate(invalid="ignore", over="ignore"):
        l2 = np.minimum(np.nan_to_num(np.abs(A * step), nan=0.0) * np.log2(np.e), 192.0)
    L = float(l2.max(initial=0.0)) * min(CHUNK, longest)
    chunks = -(-longest // CHUNK)
    return 2 * (dk + dv + 3 * CHUNK) + 8 * L + 16 * chunks + 64


# ---- norms ----------------------------------------------------------------------------------------------------------------

def rms(v, groups, eps):
    g = v.reshape(v.shape[0], groups, -1)
    return np.repeat(1 / np.sqrt((g * g).mean(-1) + eps), g.shape[2], 1)


def norm(x, w_post, z, scale, residual, w_pre, eps, groups, magnitudes=False):
    m = np.abs if magnitudes else (lambda v: v)
    u = m(x)
    if w_post is not None:
        u = u * rms(x, groups, eps) * m(w_post)
    if z is not None:
        u = u * m(silu(z))
    if scale is not None:
        u = u * m(scale)
    h = u if residual is None else u + m(residual)
    return h, None if w_pre is None else h * m(w_pre)


def norm_out(x, w_post, z, scale, residual, w_pre, eps, groups):
    h, _ = norm(x, w_post, z, scale, residual, None, eps, groups)
    return h, None if w_pre is None else h * rms(h, 1, eps) * w_pre


def _through(dy, v, w, groups, eps, m):
    """Gradients of v rms(v) w with respect to v and w; m: the identity, or magnitudes."""
    r = rms(v, groups, eps)
    n, g = m(v) * r, m(dy) * m(w)
    size = v.shape[1] // groups
    mean = np.repeat((n * g).reshape(v.shape[0], groups, size).mean(-1), size, 1)
    sign = 1 if m is np.abs else -1
    return r * (g + sign * n * mean), (m(dy) * n).sum(0)


def norm_grad(x, h, dy, dh, w_post, z, scale, w_pre, eps, groups, residual, magnitudes=False):
    m = np.abs if magnitudes else (lambda v: v)
    g, out = (m(dh) if dh is not None else np.zeros_like(x)), {}
    if w_pre is not None:
        more, out["dw_pre"] = _through(dy, x if h is None else h, w_pre, 1, eps, m)
        g = g + more
    if residual:
        out["dresidual"] = g
    u = m(x) * rms(x, groups, eps) * m(w_post) if w_post is not None else m(x)
    gate = m(silu(z)) if z is not None else 1.0
    if scale is not None:
        out["dscale"] = (g * u * gate).sum(0)
        g = g * m(scale)
    if z is not None:
        # the slope p + p z (1 - p) is a sum too, and vanishes near z = -1.28: its magnitude is that of its terms
        p = sigmoid(z)
        out["dz"] = g * u * (p + p * np.abs(z) * (1 - p) if magnitudes else silu_slope(z))
        g = g * gate
    if w_post is not None:
        g, out["dw_post"] = _through(g, x, w_post, groups, eps, m)
    out["dx"] = g
    return out
