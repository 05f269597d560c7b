"""The norms around a block against their 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import attention_util as au

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, H, F = torch.bfloat16, torch.float16, torch.float32
EPS = 1e-5

PARTS = [dict(pre=True), dict(pre=True, residual=True), dict(post=True), dict(post=True, gate=True), dict(gate=True), dict(scale=True, residual=True),
         dict(post=True, gate=True, scale=True, residual=True, pre=True)]


def _inputs(rows, d, dtype, seed, post=False, gate=False, scale=False, residual=False, pre=False, grad=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s, t=dtype: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    i = dict(x=r(rows, d), w_post=r(d, t=F) if post else None, z=r(rows, d) if gate else None, scale=r(d, t=F) if scale else None,
             residual=r(rows, d) if residual else None, w_pre=r(d, t=F) if pre else None)
    if grad:
        changed = post or gate or scale or residual
        i.update(h=r(rows, d) if changed else None, dh=r(rows, d), dy=r(rows, d) if pre else None)
    return i


def _f(i):
    return {n: au.f64(t) for n, t in i.items()}


def _roundings(d):
    """Float32 operations of a value: squares and their sum over d channels and its root (half of their error), the gate's exponential and reciprocal (8 u, and
    the argument's size, below 16), products and sums; twice for the second norm."""
    return 2 * (d / 2 + 48)


def _check(i, groups, h=None, y=None):
    f = _f(i)
    want_h, want_y = au.norm_out(f["x"], f["w_post"], f["z"], f["scale"], f["residual"], f["w_pre"], EPS, groups)
    mag, _ = au.norm(f["x"], f["w_post"], f["z"], f["scale"], f["residual"], None, EPS, groups, magnitudes=True)
    R = _roundings(f["x"].shape[1]) * au.U
    got_h, got_y = block.block_norm(**i, eps=EPS, groups=groups, h=h, y=y)
    changed = any(i[n] is not None for n in ("w_post", "z", "scale", "residual"))
    assert (got_h is i["x"]) == (not changed and h is None)
    if changed or h is not None:
        au.within(got_h, want_h, R * mag, i["x"].dtype, "h")
    if i["w_pre"] is None:
        assert got_y is None
    else:                                                                           # an error of h passes with slope rms w, and through the root, its norm's
        r = au.rms(want_h, 1, EPS)
        spread = np.abs(want_h) * r * r * np.sqrt((mag * mag).mean(1, keepdims=True))
        au.within(got_y, want_y, R * r * (mag + spread / np.maximum(r, 1e-300)) * np.abs(f["w_pre"]), i["x"].dtype, "y")
    return got_h, got_y


@pytest.mark.parametrize("parts", PARTS, ids=lambda p: "+".join(p))
@pytest.mark.parametrize("rows, d, groups", [(1, 1, 1), (3, 64, 1), (5, 96, 4), (7, 1000, 8), (2, 2048, 16), (9, 257, 1), (4, 4096, 32), (3, 63, 7)])
@pytest.mark.parametrize("dtype", [B, H, F])
def test_sizes(parts, rows, d, groups, dtype):
    _check(_inputs(rows, d, dtype, d, **parts), groups if parts.get("post") else 1)


@pytest.mark.parametrize("rows, d, groups, dtype", [(3, 16384, 1, B), (2, 16384, 128, F), (2, 16383, 1, B), (2, 8190, 3, H), (200, 4100, 1, F),
                                                    (5000, 40, 1, B), (33, 12288, 96, B)])
def test_wide_rows_and_many(rows, d, groups, dtype):
    _check(_inputs(rows, d, dtype, d, **PARTS[-1]), groups)


@pytest.mark.parametrize("dtype", [B, F])
def test_strided_rows_and_results_over_inputs(dtype):
    for shift in (0, 1):
        i = _inputs(9, 64, dtype, 3, **PARTS[-1])
        wide = torch.zeros((9, 200), device=DEV, dtype=dtype)
        for n, at in (("x", 0), ("z", 64 + shift), ("residual", 130)):
            wide[:, at:at + 64] = i[n]
            i[n] = wide[:, at:at + 64]
        before = wide.clone()
        want_h, want_y = (t.clone() for t in block.block_norm(**i, eps=EPS, groups=4))
        assert torch.equal(wide, before)
        h, y = block.block_norm(**i, eps=EPS, groups=4, h=i["residual"], y=i["x"])  # the residual stream moves on in place
        assert h is i["residual"] and torch.equal(h, want_h) and torch.equal(y, want_y)
        before[:, :64], before[:, 130:194] = want_y, want_h
        assert torch.equal(wide, before)


def test_rows_of_zeros_and_of_infinities():
    x = torch.randn((5, 96), device=DEV)
    x[1], x[3, 7] = 0, float("inf")
    _, y = block.block_norm(x, w_pre=torch.ones(96, device=DEV), eps=EPS)
    assert bool((y[1] == 0).all()) and bool(torch.isnan(y[3, 7])) and bool((y[3, :7] == 0).all()) and bool(torch.isfinite(y[[0, 2, 4]]).all())
    _, y = block.block_norm(x[1:2], w_pre=torch.ones(96, device=DEV), eps=0.0)      # 0 / 0
    assert bool(torch.isnan(y).all())


def test_leading_dimensions_and_no_rows():
    i = _inputs(12, 40, B, 5, **PARTS[-1])
    h, y = block.block_norm(**i, eps=EPS, groups=2)
    j = {n: t.reshape(3, 4, 40) if t is not None and t.dim() == 2 else t for n, t in i.items()}
    h3, y3 = block.block_norm(**j, eps=EPS, groups=2)
    assert h3.shape == (3, 4, 40) and torch.equal(h3.reshape(12, 40), h) and torch.equal(y3.reshape(12, 40), y)
    h, y = block.block_norm(x=i["x"][:0], w_pre=i["w_pre"], residual=i["residual"][:0])
    assert h.shape == y.shape == (0, 40)


def _check_gradients(i, groups, want=None, out=None):
    f = _f(i)
    residual = i["residual"] is not None
    args = (f["x"], f["h"], f["dy"], f["dh"], f["w_post"], f["z"], f["scale"], f["w_pre"], EPS, groups, residual)
    ref, mag = au.norm_grad(*args), au.norm_grad(*args, magnitudes=True)
    rows, d = f["x"].shape
    R = 2 * _roundings(d)                                                           # each norm's mean comes on top of its root
    got = block.block_norm_grad(i["x"], h=i["h"], dy=i["dy"], dh=i["dh"], w_post=i["w_post"], z=i["z"], scale=i["scale"], w_pre=i["w_pre"], eps=EPS, groups=groups,
                                residual=residual, want=want, out=out)
    assert set(got) == set(want or ref)
    for n in got:
        sums = n.startswith("dw") or n == "dscale"
        au.within(got[n], ref[n], (R + (rows if sums else 0)) * au.U * mag[n], F if sums else i["x"].dtype, n)
    return got


@pytest.mark.parametrize("parts", PARTS, ids=lambda p: "+".join(p))
@pytest.mark.parametrize("rows, d, groups", [(1, 1, 1), (3, 64, 1), (5, 96, 4), (70, 1000, 8), (300, 2048, 16), (9, 257, 1), (3, 63, 7)])
@pytest.mark.parametrize("dtype", [B, H, F])
def test_gradients(parts, rows, d, groups, dtype):
    _check_gradients(_inputs(rows, d, dtype, d, **parts, grad=True), groups if parts.get("post") else 1)


@pytest.mark.parametrize("rows, d, groups, dtype", [(3, 16384, 1, B), (2, 16384, 128, F), (2, 16383, 1, H), (400, 4100, 1, F), (5000, 40, 1, B), (900, 8192, 64, B)])
def test_gradients_of_wide_rows_and_many(rows, d, groups, dtype):
    _check_gradients(_inputs(rows, d, dtype, d, **PARTS[-1], grad=True), groups)


def test_gradients_some_wanted_in_place_and_of_no_rows():
    i = _inputs(40, 96, B, 7, **PARTS[-1], grad=True)
    every = _check_gradients(i, 4)
    for want in (["dx"], ["dz", "dw_pre"], ["dw_post", "dscale"], ["dresidual"]):
        some = _check_gradients(i, 4, want=want)
        assert all(torch.equal(some[n], every[n]) for n in want)
    dh = i["dh"]
    out = block.block_norm_grad(i["x"], h=i["h"], dy=i["dy"], dh=dh, w_post=i["w_post"], z=i["z"], scale=i["scale"], w_pre=i["w_pre"], eps=EPS, groups=4, residual=True,
                                out=dict(dresidual=dh))
    assert out["dresidual"] is dh and all(torch.equal(out[n], every[n]) for n in every)
    none = block.block_norm_grad(i["x"][:0], h=i["h"][:0], dy=i["dy"][:0], w_post=i["w_post"], w_pre=i["w_pre"])
    assert bool((none["dw_post"] == 0).all()) and bool((none["dw_pre"] == 0).all()) and none["dx"].shape == (0, 96)


def test_another_stream_and_a_captured_call():
    i = _inputs(50, 512, B, 9, **PARTS[-1], grad=True)
    forward = {n: i[n] for n in ("x", "w_post", "z", "scale", "residual", "w_pre")}
    back = dict(x=i["x"], h=i["h"], dy=i["dy"], dh=i["dh"], w_post=i["w_post"], z=i["z"], scale=i["scale"], w_pre=i["w_pre"], residual=True, groups=4)
    want, grads = block.block_norm(**forward, groups=4), block.block_norm_grad(**back)
    s = torch.cuda.Stream(device=DEV)
    torch.cuda.synchronize()
    got = block.block_norm(**forward, groups=4, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got, again = block.block_norm(**forward, groups=4), block.block_norm_grad(**back)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(again[n], grads[n]) for n in grads)
