"""Bounds on the float32 errors of a selective scan and its gradients that are carried along with the recurrences: what a state
forgets, its error forgets with it, so that a bound does not grow with the sequence.

u = 2^-24.  Every value comes with the sum of the magnitudes it is made of (H of a state, Q of a co-state) and with its error
(EH, EQ), in units of u.  To first order:

  step     D = softplus(v), v = delta + bias.  The sum is off by |v|, which moves softplus by at most |v| of itself; its exponential's argument
           |v| log2(e) by as much again; exponential, polynomial and sums by 6.  eps_D = 2 |v| + 6, or 1 without softplus.
  decay    a = 2^(D A log2(e) + c), ex2.approx off by 2^-22, the small constant c by less than 1 in units of u: 5.  The argument: eps_D, 2 for
           A log2(e), 1 for the product.  A piece of n tokens decays by 2^(A log2(e) sum D), whose sum is off by n of itself at most:
           eps_a = 5 + |D A| (eps_D + 3 + n) covers either way of going on by a token.
  state    h = a h + D x B:  EH' = a EH + eps_a a H + (eps_D + 2) |D x B| + 2 H'     (a sum, and another where pieces are joined)
  gate     silu(z) = z / (1 + exp(-z)): the exponential's argument |z|, the operations 8.  eps_z = 8 + |z|
  costate  q = C g + a q, likewise with g = dy silu(z).
Outputs add the products' own operations and those of their sums, counted where they are formed.
"""
import numpy as np

from tests import block_util as bu


def _pieces(rows, batch):
    """Additions that a sum over all tokens goes through at most: 64 tokens of a run, the runs over eight warps, those."""
    return 64 + (rows / 64 + batch) / 8 + 16


def _step_errors(delta, delta_bias, softplus):
    raw = np.abs(delta + (0 if delta_bias is None else delta_bias))
    return 2 * raw + 6 if softplus else np.ones_like(raw)


def _wide(v, d):
    return np.repeat(np.abs(v), d // v.shape[0], 0)


def _decay(step_t, eps_t, A, n):
    a = np.exp(step_t[:, None] * A)
    return a, a * (5 + np.abs(step_t[:, None] * A) * (eps_t[:, None] + 3 + n))


def _states(x, delta, A, B, delta_bias, softplus, state, seqs, piece):
    """H and EH of every token, and of the last one of every sequence."""
    rows, d = x.shape
    step, _ = bu.scan_step_sizes(delta, delta_bias, softplus)
    eps = _step_errors(delta, delta_bias, softplus)
    H, EH = np.full((rows, d, A.shape[1]), np.nan), np.full((rows, d, A.shape[1]), np.nan)
    last = np.zeros((len(seqs), d, A.shape[1]))
    for b, (lo, hi) in enumerate(seqs):
        h = np.abs(state[b]) if state is not None else np.zeros_like(last[b])
        e = np.zeros_like(h)
        for t in range(lo, hi):
            a, ea = _decay(step[t], eps[t], A, piece)
            add = np.abs(step[t] * x[t])[:, None] * _wide(B[t], d)
            e = a * e + ea * h + (eps[t][:, None] + 2) * add
            h = a * h + add
            e = e + 2 * h
            H[t], EH[t] = h, e
        last[b] = e
    return step, eps, H, EH, last


def forward(x, delta, A, B, C, D, z, delta_bias, softplus, state, seqs, piece):
    """Absolute bounds for y and the last states; `piece`: tokens of a piece at most."""
    d, n = A.shape
    _, _, H, EH, last = _states(x, delta, A, B, delta_bias, softplus, state, seqs, piece)
    skip = np.zeros(d) if D is None else np.abs(D)
    y = np.full_like(x, np.nan)
    for lo, hi in seqs:
        for t in range(lo, hi):
            c = _wide(C[t], d)
            mag = (H[t] * c).sum(1) + skip * np.abs(x[t])
            gate, eps_z = (np.abs(bu.silu(z[t])), 9 + np.abs(z[t])) if z is not None else (1.0, 0.0)
            y[t] = gate * ((EH[t] * c).sum(1) + (n + 3 + eps_z) * mag)
    return y * bu.U, last * bu.U


def gradients(dy, x, delta, A, B, C, D, z, delta_bias, softplus, state, seqs, dlast, piece):
    rows, d = x.shape
    n, groups = A.shape[1], B.shape[1]
    share = d // groups
    step, eps, H, EH, _ = _states(x, delta, A, B, delta_bias, softplus, state, seqs, piece)
    skip = np.zeros(d) if D is None else np.abs(D)
    # 1 - exp(-D) cancels down to D = 0.06, where a series takes over
    chain, eps_chain = np.ones_like(x), np.zeros_like(x)
    if softplus:
        chain = bu.scan_step_sizes(delta, delta_bias, True)[1]
        eps_chain = eps + np.where(step < 0.06, 8, 3 + 6 * np.exp(-step) / -np.expm1(-step))
    narrow = lambda v: v.reshape(groups, share, n).sum(1)  # noqa: E731
    sums = _pieces(rows, len(seqs))
    out = {k: np.full_like(x, np.nan) for k in ("dx", "ddelta", "dz")}
    out.update(dB=np.full_like(B, np.nan), dC=np.full_like(C, np.nan), dA=np.zeros_like(A), dD=np.zeros(d), ddelta_bias=np.zeros(d),
               dstate=np.zeros((len(seqs), d, n)))
    for b, (lo, hi) in enumerate(seqs):
        q = np.abs(dlast[b]) if dlast is not None else np.zeros((d, n))
        e = np.zeros_like(q)
        for t in range(hi - 1, lo - 1, -1):
            gate, eps_z = (np.abs(bu.silu(z[t])), 9 + np.abs(z[t])) if z is not None else (1.0, np.zeros(d))
            g = np.abs(dy[t]) * gate
            Bt, Ct, xt, ep = _wide(B[t], d), _wide(C[t], d), np.abs(x[t]), eps[t][:, None]
            a, ea = _decay(step[t], eps[t], A, piece)
            before = H[t - 1] if t > lo else (np.abs(state[b]) if state is not None else np.zeros((d, n)))
            e_before = EH[t - 1] if t > lo else np.zeros((d, n))
            add = Ct * g[:, None]
            q, e = q + add, e + (eps_z[:, None] + 2) * add
            e = e + 2 * q
            # sums over the channels of a group: as many operations as it has
            out["dC"][t] = narrow(EH[t] * g[:, None] + (share + 3 + eps_z[:, None]) * H[t] * g[:, None])
            dx_in = np.abs(step[t] * x[t])[:, None]
            out["dB"][t] = narrow(e * dx_in + (share + 3 + ep) * q * dx_in)
            qB, e_qB = (q * Bt).sum(1), (e * Bt).sum(1) + (n + 2) * (q * Bt).sum(1)
            out["dx"][t] = np.abs(step[t]) * (e_qB + (eps[t] + 3) * qB) + (3 + eps_z) * skip * g
            through = q * a * before
            e_through = e * a * before + q * ea * before + q * a * e_before + 3 * through
            # (A log2(e) and back: 4)
            ds = xt * qB + (through * np.abs(A)).sum(1)
            e_ds = xt * (e_qB + 2 * qB) + ((e_through + (n + 6) * through) * np.abs(A)).sum(1)
            out["ddelta"][t] = chain[t] * (e_ds + (3 + eps_chain[t]) * ds)
            out["ddelta_bias"] += out["ddelta"][t] + sums * chain[t] * ds
            out["dA"] += np.abs(step[t])[:, None] * (e_through + (ep + 2 + sums) * through)
            out["dD"] += (eps_z + 2 + sums) * g * xt
            if z is not None:
                hC = (H[t] * Ct).sum(1) + skip * xt
                e_hC = (EH[t] * Ct).sum(1) + (n + 3) * hC
                # silu'(z) = p (1 + z (1 - p)): p off by 8 + |z|, and 1 - p by what p is
                p = bu.sigmoid(z[t])
                slope, e_slope = np.abs(bu.silu_slope(z[t])), p * (1 + np.abs(z[t])) * (8 + np.abs(z[t])) + p * np.abs(z[t]) * p * (8 + np.abs(z[t]))
                out["dz"][t] = np.abs(dy[t]) * (slope * (e_hC + 3 * hC) + (e_slope + 4 * p * (1 + np.abs(z[t]))) * hC)
            e = a * e + ea * q
            q = a * q
        out["dstate"][b] = e + 2 * q
    if z is None:
        del out["dz"]
    return {k: v * bu.U for k, v in out.items()}
