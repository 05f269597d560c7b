"""The operators as a block uses them: the state space branch (projection, convolution, projections, scan, projection back onto
the residual stream) for a prompt, for single tokens behind it and for its gradients, and the control layer between projections."""
import numpy as np
import torch
import pytest

from oracle import ttc_layer as lay
from paper_2603_09221_b200 import block, lqr
from tests import block_util as bu
from tests import parity_util as pu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F, H = torch.float32, torch.float16


def _weights(g, model, d, n, rank):
    r = lambda *s, t=H: (torch.randn(s, generator=g, device=DEV) * s[-1] ** -0.5).to(t)  # noqa: E731
    return dict(w_in=r(2 * d, model), conv=r(d, 4, t=F), conv_bias=r(d, t=F), w_x=r(rank + 2 * n, d), w_dt=r(d, rank),
                dt_bias=torch.full((d,), -2.0, device=DEV), A=-torch.rand((d, n), generator=g, device=DEV) * 4 - 0.1, D=r(d, t=F), w_out=r(model, d))


def _branch(w, x, window, state, step=False):
    """y [.., model]; window and state move on in place.  Everything a backward pass wants comes along."""
    d, n = w["A"].shape
    rank = w["w_dt"].shape[1]
    xz = block.linear(x, w["w_in"])
    u, z = xz[..., :d], xz[..., d:]
    if step:
        c = block.causal_conv_step(u, w["conv"], window, w["conv_bias"], act="silu")
    else:
        c = block.causal_conv(u, w["conv"], w["conv_bias"], act="silu", state=window, state_out=window)
    p = block.linear(c, w["w_x"])
    delta = block.linear(p[..., :rank], w["w_dt"])
    args = (c, delta, w["A"], p[..., rank:rank + n], p[..., rank + n:])
    more = dict(D=w["D"], z=z, delta_bias=w["dt_bias"], softplus=True)
    if step:
        y = block.selective_scan_step(*args, **more, state=state)
    else:
        y = block.selective_scan(*args, **more, state=state, state_out=state)
    return block.linear(y, w["w_out"], residual=x), dict(u=u, z=z, c=c, p=p, delta=delta, y=y)


def _reference(w, x, window, state):
    """The same in 64 bits, autograd ready; the rounding of what passes from one operator to the next is left out."""
    f = {k: v.double() for k, v in w.items()}
    d, n = w["A"].shape
    rank = w["w_dt"].shape[1]
    xz = x @ f["w_in"].t()
    u, z = xz[..., :d], xz[..., d:]
    line = torch.cat([window, u], 1)
    c = f["conv_bias"] + sum(line[:, j:j + x.shape[1]] * f["conv"][:, j] for j in range(4))
    c = c * torch.sigmoid(c)
    p = c @ f["w_x"].t()
    step = torch.nn.functional.softplus(p[..., :rank] @ f["w_dt"].t() + f["dt_bias"])
    h, ys = state, []
    for t in range(x.shape[1]):
        h = torch.exp(step[:, t, :, None] * f["A"]) * h + (step[:, t] * c[:, t])[..., None] * p[:, t, None, rank:rank + n]
        ys.append((h * p[:, t, None, rank + n:]).sum(-1))
    y = (torch.stack(ys, 1) + f["D"] * c) * z * torch.sigmoid(z)
    return y @ f["w_out"].t() + x, h


def _close(got, want, roundings, what):
    """2-norm: every rounding to float16 on the way is off by at most 2^-11 of its value, and a value's error is passed on at
    most a few times larger (weights of unit norm, slopes near 1); four for each is allowed."""
    err = float((got.double() - want).norm() / want.norm())
    assert err <= 4 * roundings * 2.0 ** -11, (what, err)


def test_prompt_then_single_tokens():
    g = torch.Generator(device=DEV).manual_seed(1)
    model, d, n, rank, batch, tokens = 64, 96, 16, 8, 2, 37
    w = _weights(g, model, d, n, rank)
    x = torch.randn((batch, tokens + 3, model), generator=g, device=DEV).to(H)
    window, state = torch.zeros((batch, 3, d), device=DEV, dtype=H), torch.zeros((batch, d, n), device=DEV)
    want, last = _reference(w, x.double(), window.double(), state.double())
    y, _ = _branch(w, x[:, :tokens], window, state)
    ys = [y] + [_branch(w, x[:, t], window, state, step=True)[0][:, None] for t in range(tokens, tokens + 3)]
    _close(torch.cat(ys, 1), want, 6, "y")
    _close(state, last, 5, "state")


def test_gradients_of_the_branch():
    g = torch.Generator(device=DEV).manual_seed(2)
    model, d, n, rank, batch, tokens = 40, 64, 16, 8, 2, 50
    w = _weights(g, model, d, n, rank)
    x = torch.randn((batch, tokens, model), generator=g, device=DEV).to(H)
    zero = lambda *s, t=H: torch.zeros(s, device=DEV, dtype=t)  # noqa: E731
    out, k = _branch(w, x, zero(batch, 3, d), zero(batch, d, n, t=F))
    dout = torch.randn((batch, tokens, model), generator=g, device=DEV).to(H)
    # back through the branch by the gradient calls
    last = block.linear_grad(dout, k["y"], w["w_out"])
    s = block.selective_scan_grad(last["dx"], k["c"], k["delta"], w["A"], k["p"][..., rank:rank + n], k["p"][..., rank + n:], D=w["D"], z=k["z"],
                                  delta_bias=w["dt_bias"], softplus=True)
    dt = block.linear_grad(s["ddelta"], k["p"][..., :rank], w["w_dt"])
    dp = torch.cat([dt["dx"], s["dB"], s["dC"]], -1)
    px = block.linear_grad(dp, k["c"], w["w_x"])
    cv = block.causal_conv_grad(s["dx"] + px["dx"], k["u"], w["conv"], w["conv_bias"], act="silu")
    first = block.linear_grad(torch.cat([cv["dx"], s["dz"]], -1), x, w["w_in"])
    got = dict(x=first["dx"] + dout, w_in=first["dw"], conv=cv["dw"], conv_bias=cv["dbias"], w_x=px["dw"], w_dt=dt["dw"], dt_bias=s["ddelta_bias"],
               A=s["dA"], D=s["dD"], w_out=last["dw"])
    leaves = {name: v.double().requires_grad_() for name, v in dict(w, x=x).items()}
    ref, _ = _reference({name: leaves[name] for name in w}, leaves["x"], zero(batch, 3, d).double(), zero(batch, d, n).double())
    want = torch.autograd.grad((ref * dout.double()).sum(), [leaves[name] for name in got])
    for name, v in zip(got, want):
        _close(got[name], v, 14, name)


def test_control_layer_between_projections():
    """Initial state and coefficient vectors from token rows (float32 out of float16, softplus where the layer wants them
    positive), the layer, and its output back onto the residual stream."""
    g = torch.Generator(device=DEV).manual_seed(3)
    tokens, heads, n, r, model, T = 9, 4, 16, 16, 64, 8
    x = torch.randn((tokens, model), generator=g, device=DEV).to(H)
    p = lambda m, scale=1.0: (torch.randn((m, model), generator=g, device=DEV) * scale * model ** -0.5).to(H)  # noqa: E731
    names = ("s_a", "s_gamma_a", "s_gamma_b", "s_gamma_q", "s_b", "s_q", "s_qf", "r_inv", "h0")
    widths = dict.fromkeys(names, n) | dict(s_b=r, s_q=r, s_qf=r)
    plain = ("s_a", "s_b", "h0")
    weights = {k: p(heads * widths[k], 0.3) for k in names}
    vectors = {k: block.linear(x, weights[k], act="none" if k in plain else "softplus", out_dtype=F).view(tokens * heads, widths[k]) for k in names}
    L = torch.randn((r, n, n), generator=g, device=DEV) * 0.2
    B_basis, Q_basis = torch.randn((r, n, n), generator=g, device=DEV) * 0.2, L @ L.transpose(1, 2)
    solver = lqr.LqrSolver(n, n, T, (1, tokens, heads))
    u1 = torch.empty((tokens * heads, n), device=DEV)
    info = torch.empty((tokens * heads,), dtype=torch.int32, device=DEV)
    solver.solve_layer(*(vectors[k] for k in names), B_basis, Q_basis, T, u1=u1, info=info)
    w_out = (torch.randn((model, heads * n), generator=g, device=DEV) * 0.1).to(H)
    y = block.linear(u1.view(tokens, heads * n).to(H), w_out, residual=x)
    torch.cuda.synchronize()
    solver.close()
    assert int(info.abs().max()) == 0
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    for k in names:
        z = x.double() @ weights[k].double().t()
        ref = z if k in plain else torch.logaddexp(z, torch.zeros_like(z))
        # products of 64 terms and a softplus: 2 u (64 / 16 + 8) of the magnitudes, 16 u of the result
        e = 2 * bu.U * 12 * (x.double().abs() @ weights[k].double().abs().t()) * 1.13 + 16 * bu.U * (ref.abs() + z.abs())
        bu.within(vectors[k].view(tokens, -1), f64(ref), f64(e), F, k)
    ref = lay.solve_batch(*(f64(vectors[k]) for k in names), f64(B_basis), f64(Q_basis), T)
    assert pu.block_rel_err(u1.cpu().numpy(), ref["u1"], 1) <= 1e-4
    want = u1.view(tokens, heads * n).to(H).double() @ w_out.double().t() + x.double()
    e = 2 * bu.U * 12 * (u1.view(tokens, heads * n).to(H).double().abs() @ w_out.double().abs().t()) + 2 * bu.U * want.abs()
    bu.within(y, f64(want), f64(e), H, "y")


def _both(f):
    """The same call by the compiled short way (current stream) and by the long one (a stream is named): the same bits."""
    a = f(None)
    b = f(torch.cuda.current_stream())
    torch.cuda.synchronize()
    return a, b


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_both_ways_into_the_calls_for_single_tokens(dtype):
    g = torch.Generator(device=DEV).manual_seed(4)
    r = lambda *s, t=dtype: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    batch, d, n = 5, 48, 16
    wide = r(batch, 3 * d)
    for x in (r(batch, d), wide[:, d:2 * d], wide[:, 1:d + 1]):
        for bias in (None, r(d, t=F)):
            w, state = r(d, 4, t=F), r(batch, 3, d)
            states = [state.clone(), state.clone()]
            a, b = _both(lambda s: block.causal_conv_step(x, w, states[s is not None], bias, act="silu", stream=s))
            assert torch.equal(a, b) and torch.equal(*states)
        for groups in (1, 2):
            A, B, C, st = -r(d, n, t=F).abs(), r(batch, groups, n), r(batch, groups, n), r(batch, d, n, t=F)
            states = [st.clone(), st.clone()]
            out = [torch.empty_like(x), torch.empty_like(x)]
            a, b = _both(lambda s: block.selective_scan_step(x, x, A, B, C, states[s is not None], z=x, softplus=True, y=out[s is not None], stream=s))
            assert torch.equal(a, b) and torch.equal(*states) and a is out[0] and b is out[1]
    if dtype is not F:
        for rows, res in ((3, True), (200, False)):
            x, w, bias = r(rows, 2 * d)[:, 3:d + 3], r(40, d), r(40, t=F)
            a, b = _both(lambda s: block.linear(x, w, bias, act="gelu", residual=r_ if res else None, out_dtype=F, stream=s)
                         if (r_ := torch.ones((rows, 40), device=DEV)) is not None else None)
            assert torch.equal(a, b) and a.dtype == F


def test_the_short_way_refuses_what_the_long_one_refuses():
    x, w, state = torch.zeros((2, 8), device=DEV), torch.zeros((8, 4), device=DEV), torch.zeros((2, 3, 8), device=DEV)
    for bad in (dict(w=w[:7]), dict(w=w.cpu()), dict(state=state[:, :2]), dict(state=state.half()), dict(act="tanh"), dict(x=x[0]), dict(bias=w),
                dict(y=x[:1]), dict(x=x.double()), dict(act="gelu"), dict(w=torch.zeros((8, 5), device=DEV), state=torch.zeros((2, 4, 8), device=DEV))):
        with pytest.raises((ValueError, TypeError, lqr.TtcError)):
            block.causal_conv_step(**{**dict(x=x, w=w, state=state), **bad})
    A, B, st = torch.zeros((8, 4), device=DEV), torch.zeros((2, 4), device=DEV), torch.zeros((2, 8, 4), device=DEV)
    ok = dict(x=x, delta=x, A=A, B=B, C=B, state=st)
    block.selective_scan_step(**ok)
    for bad in (dict(A=A[:, :3]), dict(B=B[:1]), dict(C=B.half()), dict(state=st[0]), dict(z=x[:, :4]), dict(D=A), dict(x=x.t()), dict(delta=x.cpu())):
        with pytest.raises((ValueError, TypeError, lqr.TtcError)):
            block.selective_scan_step(**{**ok, **bad})
    h = torch.zeros((2, 8), device=DEV, dtype=H)
    for bad in (dict(w=h[:, :7]), dict(w=h.float()), dict(bias=x), dict(residual=h), dict(act="tanh"), dict(x=x), dict(out_dtype=torch.bfloat16), dict(y=h)):
        with pytest.raises((ValueError, TypeError, lqr.TtcError)):
            block.linear(**{**dict(x=h, w=torch.zeros((5, 8), device=DEV, dtype=H)), **bad})


def test_single_tokens_captured_behind_joins_copies_and_fills():
    """The kernels of single tokens are launched while what is in front of them ends: of every kind, and from two streams at once."""
    g = torch.Generator(device=DEV).manual_seed(21)
    r = lambda *s, t=H: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    w, x0, x1, taps, A = r(64, 96), r(2, 5, 96), r(2, 5, 64), r(64, 4, t=F), -torch.rand((64, 16), generator=g, device=DEV)
    x, other, window, state = r(5, 96), r(5, 64), r(5, 3, 64), r(5, 64, 16, t=F)
    first = window.clone(), state.clone()
    B = r(5, 16)

    def run():
        here, aside = torch.cuda.current_stream(), torch.cuda.Stream()
        aside.wait_stream(here)
        with torch.cuda.stream(aside):
            other.copy_(x1[0])                                       # one branch ends in a copy
        x.copy_(x0[0])                                               # so does the other
        here.wait_stream(aside)
        u = block.linear(x, w)                                       # behind a join
        c = block.causal_conv_step(u + other, taps, window, act="silu")              # behind a kernel of torch
        window[0].zero_()                                            # a fill
        y = block.selective_scan_step(c, other, A, B, B, state, softplus=True)
        return y, block.causal_conv_step(y, taps, window)

    want = [t.clone() for t in (*run(), window, state)]
    window.copy_(first[0]), state.copy_(first[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = run()
    for again in range(3):
        window.copy_(first[0]), state.copy_(first[1])
        x.zero_(), other.zero_()
        graph.replay()
        for a, b in zip((*got, window, state), want):
            assert torch.equal(a, b), again
