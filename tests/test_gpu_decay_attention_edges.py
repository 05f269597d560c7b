"""Linear attention where its chunks' tables, exponents and 16-bit operands have their limits, against the 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import attention_util as au

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, H, F = torch.bfloat16, torch.float16, torch.float32


def _inputs(tokens, heads, dk, dv, dtype, seed, groups=None):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s, t=dtype: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    return dict(q=r(1, tokens, groups or heads, dk), k=r(1, tokens, groups or heads, dk), v=r(1, tokens, heads, dv), A=-torch.rand(heads, generator=g, device=DEV) * 0.2 - 0.01,
                delta=r(1, tokens, heads).abs(), state=r(1, heads, dk, dv, t=F), dy=r(1, tokens, heads, dv), dlast=r(1, heads, dk, dv, t=F))


def _forward(i, scale=None):
    last = torch.empty_like(i["state"])
    return block.decay_attention(i["q"], i["k"], i["v"], i["A"], i["delta"], scale=scale, state=i["state"], state_out=last), last


def _grads(i, scale=None, **kw):
    return block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], scale=scale, state=i["state"], dstate_out=i["dlast"], **kw)


@pytest.mark.parametrize("dtype", [B, H])
def test_tables_of_many_chunks_are_whole(dtype):
    """Chunks whose decays differ, in walks that load the next ones meanwhile: the same bits every time."""
    i = _inputs(5000, 2, 64, 64, dtype, 3)
    i["delta"][:, ::3] = 0.01
    (y, last), grads = _forward(i), _grads(i)
    for _ in range(30):
        (y2, last2), got = _forward(i), _grads(i)
        assert torch.equal(y, y2) and torch.equal(last, last2) and all(torch.equal(got[n], grads[n]) for n in grads)
    assert block.device_error(0) == 0


def _args(i, scale):
    f = lambda n: None if i[n] is None else au.f64(i[n])[0]  # noqa: E731
    state = None if i["state"] is None else au.f64(i["state"])
    return f("q"), f("k"), f("v"), au.f64(i["A"]), f("delta"), None, False, scale, state, [(0, i["q"].shape[1])]


def _roundings(i, args):
    """As the other tests of linear attention count them, but for the arguments of exponentials: weights are zero where the sum of log2 decays between two tokens is below
    -126 (2^-126 of a product at most, which `within` leaves room for), so that no sum of more than that, with what rounding it costs, is behind a result."""
    dk, dv, tokens = args[0].shape[-1], args[2].shape[-1], args[2].shape[0]
    L = min(128 * float(np.abs(args[3] * args[4]).max()) * np.log2(np.e), 128.0)
    return 2 * (dk + dv + 3 * 128) + 8 * L + 16 * -(-tokens // 128) + 64


def _check_forward(i, scale=None):
    """y is off by the half step of each operand of 16 bits besides float32's operations, the last state by these alone."""
    args = _args(i, i["q"].shape[-1] ** -0.5 if scale is None else scale)
    R = _roundings(i, args) * au.U
    y, last = _forward(i, scale)
    want, want_last, _, _ = au.attend(*args)
    mag, mag_last, _, _ = au.attend(*args, magnitudes=True)
    au.within(y[0], want, (au.half_step(y.dtype) + R) * mag, y.dtype, "y")
    au.within(last, want_last, R * mag_last, F, "state_out")
    assert block.device_error(0) == 0


def _check_grads(i, scale=None):
    """The same of the rows' gradients, and of dstate, dA and ddelta_bias."""
    args = _args(i, i["q"].shape[-1] ** -0.5 if scale is None else scale)
    R = _roundings(i, args) * au.U
    dlast = au.f64(i["dlast"])
    ref, mag = (au.attend_grad(au.f64(i["dy"])[0], *args, dlast, magnitudes=m) for m in (False, True))
    for n, t in _grads(i, scale).items():
        rows = n in ("dq", "dk", "dv", "ddelta")
        more = 256 + (0 if rows else args[2].shape[0])
        half = au.half_step(t.dtype) if n in ("dq", "dk", "dv") else 0.0
        au.within(t[0] if rows else t, ref[n], (half + 2 * R + more * au.U) * mag[n], t.dtype, n)
    assert block.device_error(0) == 0


@pytest.mark.parametrize("strength", [1.0, 30.0, 1e4])
@pytest.mark.parametrize("dtype", [B, H])
def test_strong_decays_among_weak_ones(strength, dtype):
    i = _inputs(260, 4, 32, 32, dtype, 5)
    strong = torch.rand(1, 260, 4, generator=torch.Generator(device=DEV).manual_seed(6), device=DEV) < 0.3
    i["delta"] = torch.where(strong, i["delta"].float() * strength * 50, i["delta"].float() * 0.01).clamp(max=3e4).to(dtype)
    _check_forward(i)
    _check_grads(i)


@pytest.mark.parametrize("dtype", [B, H])
@pytest.mark.parametrize("large", [100.0, 1e4, float("inf")])
@pytest.mark.parametrize("at", [0, 32, 96])
def test_weak_decays_behind_many_that_forget_everything(dtype, large, at):
    """What passes through decays is a sum over pairs of tokens, each exp of the decays between the two whatever stands in front of them in their block: 25 tokens that forget, and
    seven that do not.  Operands are -1, 0 and 1 (keys 0 in front of the block), so that products are exact; a pair's weight is off by some 16 u (its exponential, its argument
    below 1) and passes fewer than 150 additions and products."""
    i = _inputs(at + 32, 16, 16, 16, dtype, 7)
    for n in ("q", "k", "v", "dy"):
        i[n] = i[n].round().clamp(-1, 1)
    i["k"][:, :at] = 0
    i["A"].fill_(-1.0)
    i["delta"] = i["delta"] * 0.02 + 0.01
    i["delta"][:, at:at + 25] = large
    i["state"] = i["dlast"] = None
    args = _args(i, 1.0)
    args = (*args[:4], np.minimum(args[4], 1e4), *args[5:])                       # (1e4 and infinity are the same decay)
    ref, mag = (au.attend_grad(au.f64(i["dy"])[0], *args, None, magnitudes=m) for m in (False, True))
    got = _grads(i, 1.0, want=["ddelta", "dA", "ddelta_bias"])
    for n in ("dA", "ddelta_bias"):
        au.within(got[n], ref[n], 200 * au.U * mag[n], F, n)
    au.within(got["ddelta"][0], ref["ddelta"], 200 * au.U * mag["ddelta"], dtype, "ddelta")


def _scaled(q=1.0, k=1.0, v=1.0, dy=1.0, state=0.0):
    i = _inputs(200, 2, 64, 64, H, 9)
    i.update(q=i["q"] * q, k=i["k"] * k, v=i["v"] * v, dy=i["dy"] * dy, state=i["state"] * state, dlast=i["dlast"] * state)
    return i


def _names(sizes):
    return "-".join("%s%g" % i for i in sizes.items())


@pytest.mark.parametrize("sizes", [dict(q=1e-3, k=1e-3, v=1e3), dict(q=1e-4, k=1e-4, v=3e3), dict(q=300.0, k=300.0, v=1e-3), dict(q=1e-3, k=1e3), dict(q=3e3, k=3e3, v=1e-4, scale=1e-2)],
                         ids=_names)
@pytest.mark.parametrize("state", [0.0, 1e-3, 10.0])
def test_small_and_large_products_in_float16(sizes, state):
    """Scores far below the smallest normal float16 (6e-5) and above the largest (65504), between operands and results that are neither."""
    sizes = dict(sizes)
    scale = sizes.pop("scale", None)
    i = _scaled(**sizes, state=state / sizes["q"])
    _check_forward(i, scale)


@pytest.mark.parametrize("q, state", [(1.0, 0.0), (1.0, 1e-20), (1.0, 1.0), (0.0, 1e20)])
def test_rows_that_meet_nothing_in_float16(q, state):
    """Queries and keys of zero beside others, or all queries, with states far from one."""
    i = _scaled(q=q, state=state)
    i["q"][:, 3::5], i["k"][:, :40] = 0, 0
    _check_forward(i)


@pytest.mark.parametrize("sizes", [dict(q=1e-3, k=1e-3, dy=1e3), dict(v=1e-3, dy=1e-3, q=1e-3, k=1e3), dict(v=1e-3, dy=1e-3, q=1e3, k=1e-3), dict(v=1e-4, dy=1e-3, q=1e-3, k=3e3),
                                   dict(v=300.0, dy=300.0, q=1e-3, k=1e-3), dict(q=300.0, k=300.0, v=1e-3, dy=1e-3)], ids=_names)
@pytest.mark.parametrize("state", [0.0, 1e-3, 1.0])
def test_gradients_of_small_and_large_products_in_float16(sizes, state):
    """The same of scores and of dy . v."""
    _check_grads(_scaled(**sizes, state=state))


@pytest.mark.parametrize("q, dy, state", [(1.0, 1.0, 0.0), (1.0, 1.0, 1e-20), (1.0, 1.0, 1.0), (0.0, 0.0, 1e15)])
def test_gradients_of_rows_that_meet_nothing_in_float16(q, dy, state):
    """Queries, keys, values and gradients of zero beside others, or all queries and gradients, with states far from one."""
    i = _scaled(q=q, dy=dy, state=state)
    i["q"][:, 3::5], i["dy"][:, 4::5], i["k"][:, :40], i["v"][:, 60:120], i["dlast"] = 0, 0, 0, 0, i["dlast"] * min(1.0, 1 / max(state, 1.0))
    _check_grads(i)
