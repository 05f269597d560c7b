"""Linear attention and the norms as a block uses them: norm, projections, short convolution, attention, the norm of its heads with the gate, projection, residual scale
and the next block's norm, for a prompt, for single tokens behind it and for the gradients."""
import pytest
import torch

from paper_2603_09221_b200 import block

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F, H = torch.float32, torch.float16
MODEL, HEADS, GROUPS, DK, DV, EPS = 64, 4, 2, 16, 24, 1e-5
KEYS, VALUES = GROUPS * DK, HEADS * DV


def _weights(g):
    r = lambda *s, t=H: (torch.randn(s, generator=g, device=DEV) * s[-1] ** -0.5).to(t)  # noqa: E731
    ones = lambda n: 1 + 0.1 * torch.randn(n, generator=g, device=DEV)  # noqa: E731
    return dict(w_in=r(2 * KEYS + 2 * VALUES, MODEL), w_dt=r(HEADS, MODEL), taps=r(VALUES, 4, t=F), dt_bias=torch.full((HEADS,), -1.0, device=DEV),
                A=-torch.rand(HEADS, generator=g, device=DEV) * 4 - 0.1, w_out=r(MODEL, VALUES), n_in=ones(MODEL), n_heads=ones(VALUES), n_next=ones(MODEL), scale=0.5 * ones(MODEL))


def _block(w, x, window, state, step=False):
    """The residual stream and the next block's input; window and state move on in place.  Everything a backward pass wants comes along."""
    _, n = block.block_norm(x, w_pre=w["n_in"], eps=EPS)
    p = block.linear(n, w["w_in"])
    delta = block.linear(n, w["w_dt"])
    q, k = p[..., :KEYS].unflatten(-1, (GROUPS, DK)), p[..., KEYS:2 * KEYS].unflatten(-1, (GROUPS, DK))
    u, z = p[..., 2 * KEYS:2 * KEYS + VALUES], p[..., 2 * KEYS + VALUES:]
    if step:
        v = block.causal_conv_step(u, w["taps"], window, act="silu").unflatten(-1, (HEADS, DV))
        y = block.decay_attention_step(q, k, v, w["A"], state, delta, w["dt_bias"], True)
    else:
        v = block.causal_conv(u, w["taps"], act="silu", state=window, state_out=window).unflatten(-1, (HEADS, DV))
        y = block.decay_attention(q, k, v, w["A"], delta, w["dt_bias"], True, state=state, state_out=state)
    g, _ = block.block_norm(y.flatten(-2), w_post=w["n_heads"], z=z, eps=EPS, groups=HEADS)
    o = block.linear(g, w["w_out"])
    h, out = block.block_norm(o, scale=w["scale"], residual=x, w_pre=w["n_next"], eps=EPS)
    return h, out, dict(n=n, q=q, k=k, u=u, z=z, v=v, delta=delta, y=y, g=g, o=o, h=h)


def _rms(v):
    return v / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt()


def _reference(w, x, window, state):
    """The same in 64 bits, autograd ready; the rounding of what passes from one operator to the next is left out."""
    f = {k: v.double() for k, v in w.items()}
    n = _rms(x) * f["n_in"]
    p = n @ f["w_in"].t()
    q, k = (t.unflatten(-1, (GROUPS, DK)).repeat_interleave(HEADS // GROUPS, -2) for t in (p[..., :KEYS], p[..., KEYS:2 * KEYS]))
    u, z = p[..., 2 * KEYS:2 * KEYS + VALUES], p[..., 2 * KEYS + VALUES:]
    line = torch.cat([window, u], 1)
    c = sum(line[:, j:j + x.shape[1]] * f["taps"][:, j] for j in range(4))
    v = (c * torch.sigmoid(c)).unflatten(-1, (HEADS, DV))
    a = torch.exp(f["A"] * torch.nn.functional.softplus(n @ f["w_dt"].t() + f["dt_bias"]))
    S, ys = state, []
    for t in range(x.shape[1]):
        S = a[:, t, :, None, None] * S + k[:, t, :, :, None] * v[:, t, :, None, :]
        ys.append((q[:, t, :, None, :] @ S)[:, :, 0] * DK ** -0.5)
    y = torch.stack(ys, 1)
    g = _rms(y).flatten(-2) * f["n_heads"] * z * torch.sigmoid(z)
    h = x + f["scale"] * (g @ f["w_out"].t())
    return h, _rms(h) * f["n_next"], S


def _close(got, want, roundings, what):
    """2-norm: every rounding to float16 on the way is off by at most 2^-11 of its value, and a value's error is passed on at
    most a few times larger (weights of unit norm, slopes near 1); four for each is allowed."""
    err = float((got.double() - want).norm() / want.norm())
    assert err <= 4 * roundings * 2.0 ** -11, (what, err)


def test_prompt_then_single_tokens():
    g = torch.Generator(device=DEV).manual_seed(1)
    w = _weights(g)
    batch, tokens = 2, 147                                                          # a chunk and a part of one
    x = torch.randn((batch, tokens + 3, MODEL), generator=g, device=DEV).to(H)
    window, state = torch.zeros((batch, 3, VALUES), device=DEV, dtype=H), torch.zeros((batch, HEADS, DK, DV), device=DEV)
    want_h, want_y, last = _reference(w, x.double(), window.double(), state.double())
    h, y, _ = _block(w, x[:, :tokens], window, state)
    hs, ys = [h], [y]
    for t in range(tokens, tokens + 3):
        h, y, _ = _block(w, x[:, t], window, state, step=True)
        hs.append(h[:, None]), ys.append(y[:, None])
    _close(torch.cat(hs, 1), want_h, 8, "h")
    _close(torch.cat(ys, 1), want_y, 9, "y")
    _close(state, last, 5, "state")


def test_single_tokens_captured():
    """A decoding step is one graph; what it carries moves on with every replay."""
    g = torch.Generator(device=DEV).manual_seed(2)
    w = _weights(g)
    xs = torch.randn((5, 3, MODEL), generator=g, device=DEV).to(H)
    new = lambda: (torch.zeros((3, 3, VALUES), device=DEV, dtype=H), torch.zeros((3, HEADS, DK, DV), device=DEV))  # noqa: E731
    window, state = new()
    want = [_block(w, x, window, state, step=True)[1].clone() for x in xs]
    window, state = new()
    x = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = _block(w, x, window, state, step=True)[1]
    window.zero_(), state.zero_()
    for i in range(5):
        x.copy_(xs[i])
        graph.replay()
        assert torch.equal(y, want[i])


def test_gradients():
    g = torch.Generator(device=DEV).manual_seed(3)
    w = _weights(g)
    batch, tokens = 2, 140
    x = torch.randn((batch, tokens, MODEL), generator=g, device=DEV).to(H)
    zero = lambda *s, t=H: torch.zeros(s, device=DEV, dtype=t)  # noqa: E731
    window, state = zero(batch, 3, VALUES), zero(batch, HEADS, DK, DV, t=F)
    _, _, k = _block(w, x, window.clone(), state.clone())
    dh, dout = (torch.randn((batch, tokens, MODEL), generator=g, device=DEV).to(H) for _ in range(2))
    # back through the block by the gradient calls
    e = block.block_norm_grad(k["o"], h=k["h"], dy=dout, dh=dh, scale=w["scale"], w_pre=w["n_next"], eps=EPS, residual=True)
    po = block.linear_grad(e["dx"], k["g"], w["w_out"])
    hn = block.block_norm_grad(k["y"].flatten(-2), dh=po["dx"], w_post=w["n_heads"], z=k["z"], eps=EPS, groups=HEADS)
    a = block.decay_attention_grad(hn["dx"].unflatten(-1, (HEADS, DV)), k["q"], k["k"], k["v"], w["A"], k["delta"], w["dt_bias"], True, state=state)
    cv = block.causal_conv_grad(a["dv"].flatten(-2), k["u"], w["taps"], act="silu", state=window)
    dp = torch.cat([a["dq"].flatten(-2), a["dk"].flatten(-2), cv["dx"], hn["dz"]], -1)
    pi, pd = block.linear_grad(dp, k["n"], w["w_in"]), block.linear_grad(a["ddelta"], k["n"], w["w_dt"])
    first = block.block_norm_grad(x, dy=pi["dx"] + pd["dx"], w_pre=w["n_in"], eps=EPS)
    got = dict(x=first["dx"] + e["dresidual"], w_in=pi["dw"], w_dt=pd["dw"], taps=cv["dw"], dt_bias=a["ddelta_bias"], A=a["dA"], w_out=po["dw"], n_in=first["dw_pre"],
               n_heads=hn["dw_post"], n_next=e["dw_pre"], scale=e["dscale"])
    leaves = {name: v.double().requires_grad_() for name, v in dict(w, x=x).items()}
    h, y, _ = _reference({name: leaves[name] for name in w}, leaves["x"], window.double(), state.double())
    want = torch.autograd.grad((y * dout.double()).sum() + (h * dh.double()).sum(), [leaves[name] for name in got])
    for name, v in zip(got, want):
        _close(got[name], v, 18, name)
