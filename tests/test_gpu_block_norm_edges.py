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


def test_several_threads_with_rows_of_different_widths():
    """Calls of one kernel that need more and less shared memory (123 and 61 KB), from threads that do not wait for one another: none takes the other's."""
    import threading

    lib, calls = block._load(), []
    for d in (2048, 4096) * 4:
        i = _inputs(4, d, B, d)
        out = {n: torch.empty_like(i["x"]) for n in ("dx", "dz", "dr")}
        w = {n: torch.empty_like(i["w_pre"]) for n in ("post", "scale", "pre")}
        at = lambda t: t.data_ptr()  # noqa: E731
        record = block._NORM_ARGS.pack(4, d, 16, block._type_of(i["x"]), 1e-5, at(i["x"]), at(i["z"]), 0, at(i["h"]), 0, d, d, 0, d, 0, *(at(i[n]) for n in ("w_post", "scale", "w_pre")))
        grads = block._NORM_GRADS.pack(at(i["dy"]), at(i["dh"]), *(at(t) for t in out.values()), *[d] * 5, *(at(t) for t in w.values()))
        need = lib.ttc_block_norm_grad_workspace(0, record, grads)
        calls.append((record, grads, torch.empty(need, dtype=torch.uint8, device=DEV), need, torch.cuda.Stream(device=DEV), (i, out, w)))
    torch.cuda.synchronize()
    statuses, go = [], threading.Barrier(len(calls))

    def work(record, grads, ws, need, stream, kept):
        go.wait()
        for _ in range(3000):
            status = lib.ttc_block_norm_grad(0, record, grads, ws.data_ptr(), need, stream.cuda_stream)
            if status:
                statuses.append(status)
                return

    threads = [threading.Thread(target=work, args=c) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not statuses
    i, out, w = calls[1][-1]
    _check(i, 16, 1e-5, dict(dx=out["dx"], dz=out["dz"], dresidual=out["dr"], dw_post=w["post"], dscale=w["scale"], dw_pre=w["pre"]))
