"""The bounds of scan_bounds.py, on the CPU: a recurrence in float32 stays inside of them, one that keeps its state or its
co-state in 16 bits, or loses what a piece hands on, does not."""
import numpy as np
import pytest

from tests import block_util as bu
from tests import scan_bounds as sb


def inputs(rng, tokens, d, n, groups, slow=False, gated=True):
    """Float32 values.  Memories of a few to about sixty tokens, or (slow) up to about two hundred."""
    r = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    A = -(rng.random((d, n)) * 2 + 0.05).astype(np.float32)
    bias = (0.5 * r(d) - 1).astype(np.float32)
    if slow:
        A, bias = -(rng.random((d, n)) + 0.5).astype(np.float32), (0.2 * r(d) - 4.5).astype(np.float32)
    return dict(x=r(tokens, d), delta=r(tokens, d) * np.float32(0.5 if slow else 1), A=A, B=r(tokens, groups, n), C=r(tokens, groups, n), D=r(d),
                z=r(tokens, d) if gated else None, delta_bias=bias, softplus=True, state=r(1, d, n), seqs=[(0, tokens)])


def _run(v, t, keep=lambda h: h):
    """The scan and the co-states in the type `t`, each state and co-state through `keep`; returns y, the last state and dB, dstate
    for dy = 1 and no gradient of the last state."""
    f = {k: None if a is None else a.astype(t) if isinstance(a, np.ndarray) else a for k, a in v.items()}
    one = t(1)
    raw = f["delta"] + f["delta_bias"]
    step = (np.maximum(raw, t(0)) + np.log1p(np.exp(-np.abs(raw)))).astype(t)
    gate = np.ones_like(raw) if f["z"] is None else f["z"] / (one + np.exp(-f["z"]))
    tokens, d = raw.shape
    wide = lambda u: np.repeat(u, d // u.shape[0], 0)  # noqa: E731
    h, ys = f["state"][0], []
    for i in range(tokens):
        h = keep((np.exp(step[i][:, None] * f["A"]) * h + (step[i] * f["x"][i])[:, None] * wide(f["B"][i])).astype(t))
        ys.append(((h * wide(f["C"][i])).sum(1) + f["D"] * f["x"][i]) * gate[i])
    q, dB = np.zeros_like(h), np.zeros_like(f["B"])
    for i in range(tokens - 1, -1, -1):
        q = keep((q + wide(f["C"][i]) * gate[i][:, None]).astype(t))
        dB[i] = (q * (step[i] * f["x"][i])[:, None]).reshape(dB.shape[1], -1, q.shape[1]).sum(1)
        q = (np.exp(step[i][:, None] * f["A"]) * q).astype(t)
    return np.stack(ys), h, dB, q


def _over(v, got):
    """How far each output is over its bound (1: at it), and the relative errors in the 2-norm."""
    f = {k: None if a is None else a.astype(np.float64) if isinstance(a, np.ndarray) else a for k, a in v.items()}
    want, last, _ = bu.scan(**f)
    ey, el = sb.forward(**f, piece=128)
    ones = np.ones_like(f["x"])
    g, eg = bu.scan_grad(ones, **f, dlast=None), sb.gradients(ones, **f, dlast=None, piece=16)
    pairs = [(got[0], want, ey), (got[1], last[0], el[0]), (got[2], g["dB"], eg["dB"]), (got[3], g["dstate"][0], eg["dstate"][0])]
    return [float((np.abs(a - b) / e).max()) for a, b, e in pairs], [float(np.linalg.norm(a - b) / np.linalg.norm(b)) for a, b, _ in pairs]


SHAPES = [(1025, 8, 16, 1), (700, 3, 4, 1), (513, 40, 64, 2)]


@pytest.mark.parametrize("slow", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_float32_is_inside_and_sixteen_bits_are_not(shape, slow):
    rng = np.random.default_rng(7)
    v = inputs(rng, *shape, slow=slow)
    over, off = _over(v, _run(v, np.float32))
    assert max(over) < 1 and max(off) < 1e-5, (over, off)
    for keep in (lambda h: h.astype(np.float16).astype(np.float32), lambda h: (h.view(np.uint32) + 0x1000 & 0xffffe000).view(np.float32)):
        over, off = _over(v, _run(v, np.float32, keep))             # 11 bits each: float16, and float32 cut down to as many
        assert min(off) > 1e-5, off
        if not slow:
            assert min(over) > 1, over


def test_a_lost_share_of_a_piece_is_outside():
    rng = np.random.default_rng(8)
    v = inputs(rng, 513, 8, 16, 1, slow=True)
    good = _run(v, np.float64)
    calls = [0]

    def lose(h):                                                     # once, in the middle of the walk: a thousandth of the state
        calls[0] += 1
        return h * (1 - 1e-3) if calls[0] % 513 == 490 else h

    over, off = _over(v, _run(v, np.float64, lose))
    assert max(_over(v, good)[0]) < 1e-6 and over[1] > 1 and off[1] > 1e-5, (over, off)
