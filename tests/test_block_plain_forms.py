"""The plain forms of block_util.py: their gradients against differences of their forward passes, on the CPU."""
import numpy as np
import pytest

from tests import block_util as bu


def _numbers(rng, *shape):
    return rng.standard_normal(shape)


def _check(loss, grads, inputs, rng, eps=1e-6):
    """Central differences along a random direction of every input; eps^2 and 1e-16 / eps leave about 1e-9 of the values."""
    for name, v in inputs.items():
        way = _numbers(rng, *v.shape)
        with np.errstate(all="raise"):
            up, down = (loss(**{**inputs, name: v + s * eps * way}) for s in (1, -1))
        want = (up - down) / (2 * eps)
        got = float((grads[name] * way).sum())
        assert abs(got - want) <= 1e-7 * (1 + np.abs(grads[name] * way).sum()), (name, got, want)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("taps", [2, 4])
def test_convolution(act, taps):
    rng = np.random.default_rng(3)
    seqs = [(0, 5), (5, 5), (5, 6), (6, 8)]
    ins = dict(x=_numbers(rng, 8, 3), w=_numbers(rng, 3, taps), bias=_numbers(rng, 3), state=_numbers(rng, 4, taps - 1, 3))
    dy, dlast = _numbers(rng, 8, 3), _numbers(rng, 4, taps - 1, 3)

    def loss(x, w, bias, state):
        y, last, _ = bu.conv(x, w, bias, act, state, seqs)
        return (y * dy).sum() + (last * dlast).sum()

    g = bu.conv_grad(dy, ins["x"], ins["w"], ins["bias"], act, ins["state"], seqs, dlast)
    _check(loss, {"x": g["dx"], "w": g["dw"], "bias": g["dbias"], "state": g["dstate"]}, ins, rng)


@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("gated", [True, False])
def test_scan(softplus, gated):
    rng = np.random.default_rng(4)
    seqs = [(0, 5), (5, 5), (5, 6), (6, 9)]
    d, n = 4, 3
    ins = dict(x=_numbers(rng, 9, d), delta=np.abs(_numbers(rng, 9, d)), A=-np.abs(_numbers(rng, d, n)), B=_numbers(rng, 9, 2, n),
               C=_numbers(rng, 9, 2, n), D=_numbers(rng, d), delta_bias=np.abs(_numbers(rng, d)), state=_numbers(rng, 4, d, n))
    if gated:
        ins["z"] = _numbers(rng, 9, d)
    dy, dlast = _numbers(rng, 9, d), _numbers(rng, 4, d, n)

    def loss(z=None, **v):
        y, last, _ = bu.scan(z=z, softplus=softplus, seqs=seqs, **v)
        return (y * dy).sum() + (last * dlast).sum()

    g = bu.scan_grad(dy, z=ins.get("z"), softplus=softplus, seqs=seqs, dlast=dlast, **{k: v for k, v in ins.items() if k != "z"})
    _check(loss, {k[1:]: v for k, v in g.items()}, ins, rng)
