"""The 64-bit forms that the kernels are held to, against automatic differentiation and differences (no GPU needed)."""
import numpy as np
import torch

from tests import attention_util as au

SEQS = [(0, 5), (5, 5), (5, 12)]


def _inputs(seed, rows=12, heads=4, groups=2, dk=3, dv=5):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    return dict(q=r(rows, groups, dk), k=r(rows, groups, dk), v=r(rows, heads, dv), A=-r(heads).abs() - 0.1, delta=r(rows, heads), bias=r(heads), dy=r(rows, heads, dv),
                state=r(3, heads, dk, dv), dlast=r(3, heads, dk, dv))


def _recurrence(i, scale):
    """With the decays as a product over the tokens between two, instead of a state."""
    rows, heads, _ = i["v"].shape
    share = heads // i["q"].shape[1]
    q, k = i["q"].repeat_interleave(share, 1) * scale, i["k"].repeat_interleave(share, 1)
    l = i["A"] * torch.nn.functional.softplus(i["delta"] + i["bias"])
    ys, last = [], []
    for b, (lo, hi) in enumerate(SEQS):
        G = torch.cumsum(l[lo:hi], 0)
        S = torch.exp(G[-1])[:, None, None] * i["state"][b] if hi > lo else i["state"][b]
        for t in range(lo, hi):
            at = t - lo
            w = torch.exp(G[at] - G[:at + 1])                                       # [tokens, heads]
            scores = torch.einsum("hk,thk->th", q[t], k[lo:t + 1]) * w
            ys.append(torch.einsum("th,thv->hv", scores, i["v"][lo:t + 1]) + torch.exp(G[at])[:, None] * torch.einsum("hk,hkv->hv", q[t], i["state"][b]))
        for t in range(lo, hi):
            S = S + torch.exp(G[-1] - G[t - lo])[:, None, None] * k[t][:, :, None] * i["v"][t][:, None, :]
        last.append(S)
    return torch.stack(ys), torch.stack(last)


def test_attention_and_its_gradients_against_autograd():
    i = _inputs(3)
    leaves = {n: t.clone().requires_grad_() for n, t in i.items()}
    y, last = _recurrence(leaves, 0.7)
    grads = torch.autograd.grad((y * i["dy"]).sum() + (last * i["dlast"]).sum(), [leaves[n] for n in ("q", "k", "v", "delta", "A", "bias", "state")])
    n = {k: t.numpy() for k, t in i.items()}
    args = (n["q"], n["k"], n["v"], n["A"], n["delta"], n["bias"], True, 0.7, n["state"], SEQS)
    got = au.attend(*args)
    np.testing.assert_allclose(got[0], y.detach().numpy(), atol=1e-12)
    np.testing.assert_allclose(got[1], last.detach().numpy(), atol=1e-12)
    back = au.attend_grad(n["dy"], *args, n["dlast"])
    for name, want in zip(("dq", "dk", "dv", "ddelta", "dA", "ddelta_bias", "dstate"), grads):
        np.testing.assert_allclose(back[name], want.numpy(), atol=1e-11, err_msg=name)


def test_gradient_of_the_decays_against_differences():
    n = {k: t.numpy() for k, t in _inputs(4).items()}
    loss = lambda delta, A: sum((a * b).sum() for a, b in zip(au.attend(n["q"], n["k"], n["v"], A, delta, n["bias"], False, 0.5, n["state"], SEQS)[:2],  # noqa: E731
                                                              (n["dy"], n["dlast"])))
    back = au.attend_grad(n["dy"], n["q"], n["k"], n["v"], n["A"], n["delta"], n["bias"], False, 0.5, n["state"], SEQS, n["dlast"])
    e = 1e-6
    for at in ((0, 0), (4, 1), (5, 2), (11, 3)):
        d = np.zeros_like(n["delta"])
        d[at] = e
        np.testing.assert_allclose((loss(n["delta"] + d, n["A"]) - loss(n["delta"] - d, n["A"])) / (2 * e), back["ddelta"][at], rtol=1e-6, atol=1e-6)
    d = np.zeros_like(n["A"])
    d[1] = e
    np.testing.assert_allclose((loss(n["delta"], n["A"] + d) - loss(n["delta"], n["A"] - d)) / (2 * e), back["dA"][1], rtol=1e-6, atol=1e-6)


def test_norms_against_autograd():
    g = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    x, z, res, dh, dy = (r(7, 12) for _ in range(5))
    wp, s, w = r(12), r(12), r(12)
    leaves = [t.clone().requires_grad_() for t in (x, z, res, wp, s, w)]
    lx, lz, lr, lp, ls, lw = leaves
    m = lx.reshape(7, 3, 4)
    u = (m / (m.pow(2).mean(-1, keepdim=True) + 1e-3).sqrt()).reshape(7, 12) * lp * torch.nn.functional.silu(lz)
    h = lr + ls * u
    y = h / (h.pow(2).mean(-1, keepdim=True) + 1e-3).sqrt() * lw
    want = torch.autograd.grad((h * dh).sum() + (y * dy).sum(), leaves)
    n = lambda t: t.numpy()  # noqa: E731
    gh, gy = au.norm_out(n(x), n(wp), n(z), n(s), n(res), n(w), 1e-3, 3)
    np.testing.assert_allclose(gh, h.detach().numpy(), atol=1e-12)
    np.testing.assert_allclose(gy, y.detach().numpy(), atol=1e-12)
    got = au.norm_grad(n(x), gh, n(dy), n(dh), n(wp), n(z), n(s), n(w), 1e-3, 3, True)
    for name, v in zip(("dx", "dz", "dresidual", "dw_post", "dscale", "dw_pre"), want):
        np.testing.assert_allclose(got[name], v.numpy(), atol=1e-11, err_msg=name)
