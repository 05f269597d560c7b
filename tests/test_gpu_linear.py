"""Projections with bias, activation and residual, and their gradients, against 64-bit products.

Bounds: u = 2^-24.  The tensor cores add products of 16-bit numbers (exact in float32) in steps of 16 contraction indices to a
float32 accumulator that is cut off rather than rounded (2 u of the magnitudes' sum at each step, and once more within a
step); sums of parts and of the few-rows kernel's warps are covered by the same count: 2 u (k / 16 + 8) S, S the product of
magnitudes.  Activations have slopes of at most 1.13 and errors below 16 u of the result and of z."""
import numpy as np
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import block_util as bu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = torch.float32
ACTS = ["none", "relu", "silu", "gelu", "softplus"]


def _act(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * torch.special.ndtr(z),
            "softplus": lambda: torch.logaddexp(z, torch.zeros_like(z))}[act]()


def _randn(g, *s, t=torch.bfloat16):
    return torch.randn(s, generator=g, device=DEV).to(t)


def _bound(x, w, k):
    return 2 * bu.U * (k / 16 + 8) * (x.abs().double() @ w.abs().double().t())


def _check(x, w, bias=None, act="none", residual=None, out_dtype=None, pre=False, y=None):
    k = w.shape[1]
    out_dtype = out_dtype or x.dtype
    xx = x.reshape(-1, k)
    p = torch.full((*x.shape[:-1], w.shape[0]), 9.0, device=DEV, dtype=x.dtype) if pre else None
    keep = None if residual is None else residual.clone()
    got = block.linear(x, w, bias, act=act, residual=residual, out_dtype=out_dtype, pre=p, y=y)
    z = xx.double() @ w.double().t()
    e = _bound(xx, w, k)
    if bias is not None:
        z, e = z + bias.double(), e + bu.U * (z.abs() + bias.double().abs())
    if pre:
        bu.within(p.reshape(z.shape), z.cpu().numpy(), e.cpu().numpy(), x.dtype, "pre")
    a = _act(z, act)
    if act != "none":
        e = 1.13 * e + 16 * bu.U * (a.abs() + z.abs())
    if keep is not None:
        a = a + keep.reshape(z.shape).double()
        e = e + bu.U * a.abs()
    bu.within(got.reshape(z.shape), a.cpu().numpy(), e.cpu().numpy(), out_dtype, "y")
    assert block.device_error(0) == 0
    return got


# rows, k, m: one row, few rows, tiles, parts of the contraction, odd sizes whose rows TMA cannot read
SHAPES = [(1, 64, 16), (1, 7, 1), (5, 100, 33), (8, 256, 64), (17, 512, 130), (32, 1000, 48), (33, 64, 64), (100, 24, 300), (128, 64, 256), (129, 520, 257),
          (300, 4096, 96), (257, 99, 101), (1000, 1024, 1032), (64, 8192, 64), (2048, 128, 4096)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, out, dtype):
    rows, k, m = shape
    g = torch.Generator(device=DEV).manual_seed(1)
    _check(_randn(g, rows, k, t=dtype), _randn(g, m, k, t=dtype), _randn(g, m, t=F), out_dtype=F if out == "f32" else dtype)


@pytest.mark.parametrize("rows", [1, 8, 9, 16, 17, 32, 33, 57, 64, 65])
@pytest.mark.parametrize("k, m", [(1024, 33), (2064, 50), (4100, 30), (5003, 17), (9000, 1000)])
def test_few_rows_over_long_contractions(rows, k, m):
    """The contraction shared out between the blocks of a cluster, in parts that end anywhere."""
    g = torch.Generator(device=DEV).manual_seed(rows + k)
    _check(_randn(g, rows, k), _randn(g, m, k), _randn(g, m, t=F), out_dtype=F if rows % 2 else torch.bfloat16)


@pytest.mark.parametrize("rows, k, m", [(3, 64, 40), (200, 136, 200), (150, 2048, 65), (90, 33, 77)])
@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_activations_with_residual_and_pre(act, out, rows, k, m):
    g = torch.Generator(device=DEV).manual_seed(2)
    t = torch.bfloat16
    o = F if out == "f32" else t
    x, w, b, r = _randn(g, rows, k), _randn(g, m, k) * k ** -0.5, _randn(g, m, t=F), _randn(g, rows, m, t=o)
    got = _check(x, w * 3, b, act, r, o, pre=True)
    same = r.clone()
    assert torch.equal(block.linear(x, w * 3, b, act=act, residual=same, y=same), got)            # in place on the residual stream
    _check(x, w, None, act)


def test_leading_dimensions_slices_and_one_row():
    g = torch.Generator(device=DEV).manual_seed(3)
    wide = _randn(g, 4, 30, 200)
    for lo, hi in ((0, 64), (8, 72), (1, 100), (100, 200)):
        _check(wide[..., lo:hi], _randn(g, 70, hi - lo))
    w = _randn(g, 96, 300)
    _check(_randn(g, 60, 128), w[:80, 3:131])                                                     # W as a slice
    out = torch.full((120, 100), 5.0, device=DEV, dtype=torch.bfloat16)
    for lo in (0, 3):
        _check(_randn(g, 120, 64), _randn(g, 40, 64), y=out[:, lo:lo + 40])
        assert bool((out[:, lo + 40:] == 5).all())
    _check(_randn(g, 64), _randn(g, 24, 64))


def test_values_that_are_no_numbers_stay_in_their_rows():
    g = torch.Generator(device=DEV).manual_seed(4)
    for rows in (6, 200):
        x, w = _randn(g, rows, 96), _randn(g, 80, 96)
        x[2, 5] = float("nan")
        x[4, 7] = float("inf")
        for act in ("none", "relu"):
            y = block.linear(x, w, act=act)
            assert torch.isnan(y[2]).all()
            good = [i for i in range(rows) if i not in (2, 4)]
            assert torch.isfinite(y[good]).all()


def _check_grad(x, w, dy, act, pre):
    got = block.linear_grad(dy, x, w, act=act, pre=pre)
    k, m = x.shape[-1], w.shape[0]
    xx, dd = x.reshape(-1, k).double(), dy.reshape(-1, m).double()
    rows, ww = xx.shape[0], w.double()
    if pre is None:
        dz, slope_e = dd, torch.zeros_like(dd)
    else:
        z = pre.reshape(-1, m).double().requires_grad_()
        (dz,) = torch.autograd.grad(_act(z, act), z, dd)
        slope_e = 32 * bu.U * dd.abs() * (1 + z.detach().abs())
    exact_dz = pre is None and dy.dtype == x.dtype
    half = 0.0 if exact_dz else bu.half_step(x.dtype)
    tiny = 2.0 ** -25 if x.dtype == torch.float16 and not exact_dz else 0.0                       # dZ below float16's numbers
    ez = half * dz.abs() + (1 + half) * slope_e + tiny                                            # of the 16-bit dZ
    n = lambda t: t.detach().cpu().numpy()  # noqa: E731
    e = ez @ ww.abs() + 2 * bu.U * (m / 16 + 8) * (dz.abs() @ ww.abs()) * (1 + 2 * half)
    bu.within(got["dx"].reshape(rows, k), n(dz @ ww), n(e), x.dtype, "dx")
    e = ez.t() @ xx.abs() + 2 * bu.U * (rows / 16 + 8) * (dz.abs().t() @ xx.abs()) * (1 + 2 * half)
    bu.within(got["dw"], n(dz.t() @ xx), n(e), x.dtype, "dw")
    bu.within(got["dbias"], n(dz.sum(0)), n(slope_e.sum(0) + (rows + 8) * bu.U * dz.abs().sum(0)), F, "dbias")
    assert block.device_error(0) == 0
    return got


GRAD_SHAPES = [(1, 8, 16), (3, 33, 7), (40, 64, 128), (129, 100, 257), (700, 256, 64), (5000, 64, 72), (1030, 136, 1000), (4096, 16, 8)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", GRAD_SHAPES)
def test_gradients(shape, dtype):
    rows, k, m = shape
    g = torch.Generator(device=DEV).manual_seed(5)
    _check_grad(_randn(g, rows, k, t=dtype), _randn(g, m, k, t=dtype), _randn(g, rows, m, t=dtype), "none", None)


@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("act", ACTS[1:])
def test_gradients_of_activations(act, out):
    g = torch.Generator(device=DEV).manual_seed(6)
    for rows, k, m in ((2, 40, 24), (333, 72, 200), (64, 65, 33)):
        _check_grad(_randn(g, rows, k), _randn(g, m, k), _randn(g, rows, m, t=F if out == "f32" else torch.bfloat16), act, _randn(g, rows, m))


def test_gradients_of_a_float32_output_and_of_slices():
    g = torch.Generator(device=DEV).manual_seed(7)
    _check_grad(_randn(g, 100, 64), _randn(g, 48, 64), _randn(g, 100, 48, t=F), "none", None)
    wide, wd = _randn(g, 2, 50, 160), _randn(g, 100, 96)
    _check_grad(wide[..., 3:67], wd[:, 5:69], _randn(g, 2, 50, 100), "none", None)


def test_parts_of_the_gradients_and_no_rows():
    g = torch.Generator(device=DEV).manual_seed(8)
    x, w, dy = _randn(g, 50, 64), _randn(g, 48, 64), _randn(g, 50, 48)
    whole = block.linear_grad(dy, x, w)
    for k in whole:
        one = block.linear_grad(dy, x, w, want=(k,))
        assert set(one) == {k} and torch.equal(one[k], whole[k])
    none = block.linear_grad(dy[:0], x[:0], w)
    assert not none["dw"].any() and not none["dbias"].any() and none["dx"].shape == (0, 64)
    assert block.linear(x[:0], w).shape == (0, 48)


def test_gradient_against_differences():
    """Float16 with steps and values that are exact, so that the product's change is the gradient's."""
    x = torch.randint(-3, 4, (40, 64), device=DEV).half()
    w = torch.randint(-3, 4, (24, 64), device=DEV).half()
    dy = torch.randint(-3, 4, (40, 24), device=DEV).half()
    got = block.linear_grad(dy, x, w)
    loss = lambda x_, w_: float((block.linear(x_, w_, out_dtype=F).double() * dy.double()).sum())  # noqa: E731
    for i, j in ((0, 0), (39, 63), (17, 5)):
        up = x.clone()
        up[i, j] += 1
        assert loss(up, w) - loss(x, w) == float(got["dx"][i, j])
    for i, j in ((0, 0), (23, 63), (11, 30)):
        up = w.clone()
        up[i, j] += 1
        assert loss(x, up) - loss(x, w) == float(got["dw"][i, j])


def test_pairs_of_ctas_in_a_graph():
    """Enough tiles of 256 x 256 for two CTAs on each, ragged in both directions; captured and replayed on new values."""
    g = torch.Generator(device=DEV).manual_seed(10)
    x, w, b, r = _randn(g, 9001, 72), _randn(g, 1000, 72), _randn(g, 1000, t=F), _randn(g, 9001, 1000)
    first = _check(x, w, b, "silu", r)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block.linear(x, w, b, act="silu", residual=r)
    graph.replay()
    assert torch.equal(y, first)
    x.copy_(_randn(g, 9001, 72))
    graph.replay()
    assert torch.equal(y, _check(x, w, b, "silu", r))
    _check_grad(_randn(g, 1024, 3000), _randn(g, 9000, 3000), _randn(g, 1024, 9000), "relu", _randn(g, 1024, 9000))


def test_long_contractions_in_float32():
    """Added up in segments of 512 indices, 32 steps of the tensor cores, each of which cuts off u of the partial sum in the mean.  With
    random signs a partial sum is in the mean not larger than the segment's own, so a segment is off by at most 32 u = 1.9e-6 of
    its norm, and the segments' norms add up in squares to the result's."""
    g = torch.Generator(device=DEV).manual_seed(11)
    for rows, k, m in ((1500, 4096, 700), (64, 8000, 96), (20, 4096, 50), (300, 1100, 257)):
        x, w = _randn(g, rows, k), _randn(g, m, k)
        y = _check(x, w, out_dtype=F)
        want = x.double() @ w.double().t()
        assert float((y.double() - want).norm() / want.norm()) <= 32 * bu.U


def test_graphs_and_streams():
    g = torch.Generator(device=DEV).manual_seed(9)
    x, w, b, dy = _randn(g, 70, 1033), _randn(g, 90, 1033), _randn(g, 90, t=F), _randn(g, 70, 90)
    y, grads = block.linear(x, w, b, act="silu"), block.linear_grad(dy, x, w)
    kept, graphs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept.append((block.linear(x, w, b, act="silu"), block.linear_grad(dy, x, w)))
        graphs.append(graph)
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for again, gg in kept:
            assert torch.equal(again, y) and all(torch.equal(gg[k], grads[k]) for k in grads)
    other = block.linear(x, w, b, act="silu", stream=side)
    side.synchronize()
    assert torch.equal(other, y)
