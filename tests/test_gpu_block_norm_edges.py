"""Gradients of the norms where their kernels' sums meet: one group over rows of several warps."""
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import attention_util as au

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, H, F = torch.bfloat16, torch.float16, torch.float32


def _inputs(rows, d, dtype, seed, scale=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s, t=dtype: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    return dict(x=r(rows, d), h=r(rows, d), dy=r(rows, d), dh=r(rows, d), w_post=r(d, t=F), z=r(rows, d), scale=r(d, t=F) if scale else None, w_pre=r(d, t=F))


def _check(i, groups, eps, got):
    """Float32 operations of a value as in the tests of the norms: two norms, each with its mean on top of its root; the parameters' gradients are sums over the rows."""
    f = {n: au.f64(t) for n, t in i.items()}
    args = (f["x"], f["h"], f["dy"], f["dh"], f["w_post"], f["z"], f["scale"], f["w_pre"], eps, groups, True)
    ref, mag = au.norm_grad(*args), au.norm_grad(*args, magnitudes=True)
    rows, d = f["x"].shape
    assert set(got) == set(ref)
    for n in got:
        sums = n.startswith("dw") or n == "dscale"
        au.within(got[n], ref[n], (4 * (d / 2 + 48) + (rows if sums else 0)) * au.U * mag[n], F if sums else i["x"].dtype, n)


@pytest.mark.parametrize("rows, d, dtype", [(700, 2048, B), (700, 2048, F), (500, 4096, H), (333, 777, B), (160, 16384, B), (160, 16383, F)])
def test_one_group_and_the_next_norm_over_many_warps(rows, d, dtype):
    """Sums of one value and of two take turns in every row: the same bits every time."""
    i = _inputs(rows, d, dtype, d)
    first = block.block_norm_grad(**i, eps=1e-5, residual=True)
    _check(i, 1, 1e-5, first)
    for _ in range(30):
        got = block.block_norm_grad(**i, eps=1e-5, residual=True)
        assert all(torch.equal(got[n], first[n]) for n in first)


@pytest.mark.parametrize("rows", [1, 5, 149, 600, 1187])
@pytest.mark.parametrize("d, groups, dtype", [(64, 1, F), (96, 4, B), (1000, 8, F), (257, 1, H), (2048, 16, B), (2048, 1, B)])
def test_no_eps(rows, d, groups, dtype):
    """With an eps of nothing, rows that are not there (the last round of a kernel's workers) leave the parameters' gradients alone."""
    i = _inputs(rows, d, dtype, rows)
    _check(i, groups, 0.0, block.block_norm_grad(**i, eps=0.0, groups=groups, residual=True))
