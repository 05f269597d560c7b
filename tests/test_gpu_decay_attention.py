"""Linear attention with a decay for each head against its 64-bit form, token by token."""
import numpy as np
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import attention_util as au

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, H, F = torch.bfloat16, torch.float16, torch.float32


def _inputs(lead, batch, heads, groups, dk, dv, dtype, seed, decay="token", strength=1.0, state=True, offsets=None, grad=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s, t=dtype, a=1.0: (torch.randn(s, generator=g, device=DEV) * a).to(t)  # noqa: E731
    i = dict(q=r(*lead, groups, dk), k=r(*lead, groups, dk), v=r(*lead, heads, dv), A=-torch.rand(heads, generator=g, device=DEV) * strength - 1e-3,
             delta=r(*lead, heads, a=0.5) if decay == "token" else None, delta_bias=r(heads, t=F, a=0.5) if decay == "token" else None,
             softplus=decay == "token", state=r(batch, heads, dk, dv, t=F, a=0.3) if state else None,
             offsets=torch.tensor(offsets, dtype=torch.int32, device=DEV) if offsets is not None else None)
    if grad:
        i.update(dy=r(*lead, heads, dv), dlast=r(batch, heads, dk, dv, t=F) if state else None)
    return i


def _flat(t, lead):
    return None if t is None else au.f64(t).reshape(int(np.prod(lead)), *t.shape[len(lead):])


def _args(i, lead, scale):
    f = lambda n: _flat(i[n], lead)  # noqa: E731
    seqs = au.spans(lead, i["offsets"].tolist() if i["offsets"] is not None else None)
    return (f("q"), f("k"), f("v"), au.f64(i["A"]), f("delta"), au.f64(i["delta_bias"]), i["softplus"], scale, au.f64(i["state"]), seqs)


def _bounds(i, args, lead):
    heads, dk, dv = i["v"].shape[-2], i["q"].shape[-1], i["v"].shape[-1]
    longest = max((hi - lo for lo, hi in args[-1]), default=0)
    return au.roundings(dk, dv, longest, args[3], args[4], args[5], args[6], args[2].shape[0], heads) * au.U, -(-longest // au.CHUNK)


def _call(i, scale=None, **kw):
    return block.decay_attention(i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], i["softplus"], scale, i["state"], i["offsets"], **kw)


def _check_forward(i, lead, scale=None, y=None, state_out=None):
    s = i["q"].shape[-1] ** -0.5 if scale is None else scale
    args = _args(i, lead, s)
    want, last, _, _ = au.attend(*args)
    mag, mag_last, _, _ = au.attend(*args, magnitudes=True)
    rel, _ = _bounds(i, args, lead)
    batch = len(args[-1])
    if state_out is None:
        state_out = torch.full((batch, i["v"].shape[-2], i["q"].shape[-1], i["v"].shape[-1]), float("nan"), device=DEV)
    if y is None:
        y = torch.full_like(i["v"], float("nan"))
    assert _call(i, scale, y=y, state_out=state_out) is y
    inside = np.zeros(want.shape[0], bool)
    for lo, hi in args[-1]:
        inside[lo:hi] = True
    got = y.reshape(want.shape)[torch.from_numpy(inside).to(DEV)]
    au.within(got, want[inside], ((au.half_step(y.dtype) + rel) * mag)[inside], y.dtype, "y")
    assert bool(torch.isnan(y.reshape(want.shape)[torch.from_numpy(~inside).to(DEV)]).all())           # rows of no sequence
    au.within(state_out, last, rel * mag_last, F, "state_out")
    assert block.device_error(0) == 0


@pytest.mark.parametrize("tokens", [1, 2, 31, 32, 33, 127, 128, 129, 257, 600])
@pytest.mark.parametrize("dk, dv, dtype", [(64, 64, B), (128, 128, B), (128, 64, H), (64, 128, H), (16, 128, B)])
def test_lengths(tokens, dk, dv, dtype):
    lead = (2, tokens)
    _check_forward(_inputs(lead, 2, 2, 1, dk, dv, dtype, tokens), lead)


@pytest.mark.parametrize("dk, dv", [(1, 1), (7, 3), (8, 72), (36, 20), (72, 8), (65, 127), (127, 65), (100, 100)])
@pytest.mark.parametrize("dtype", [B, H])
def test_widths_of_heads(dk, dv, dtype):
    lead = (2, 150)
    _check_forward(_inputs(lead, 2, 3, 3, dk, dv, dtype, dk), lead)


@pytest.mark.parametrize("heads, groups", [(1, 1), (6, 2), (8, 1), (4, 4)])
@pytest.mark.parametrize("decay", ["token", "head"])
def test_heads_and_decays(heads, groups, decay):
    lead = (1, 200)
    _check_forward(_inputs(lead, 1, heads, groups, 32, 48, B, heads, decay, state=False), lead, scale=-1.5)


@pytest.mark.parametrize("offsets, rows", [([0, 0, 130, 130, 131, 400], 400), ([3, 60, 60, 64, 199], 210), ([0, 300], 300), ([5], 9), ([0, 1, 2, 3, 4], 4),
                                           ([0] + [7 * i for i in range(1, 41)], 280)])
@pytest.mark.parametrize("dk, dtype", [(64, B), (40, H), (20, B)])
def test_packed_sequences_some_empty_and_rows_of_none(offsets, rows, dk, dtype):
    _check_forward(_inputs((rows,), len(offsets) - 1, 4, 2, dk, 64, dtype, rows, offsets=offsets), (rows,))


def test_few_heads_are_cut_into_pieces():
    """One sequence of one head is walked along in as many pieces as there are SMs."""
    lead = (1, 3000)
    i = _inputs(lead, 1, 1, 1, 64, 32, B, 7, strength=0.05)
    _check_forward(i, lead)
    i["offsets"], flat = torch.tensor([0, 10, 10, 2600, 3000], dtype=torch.int32, device=DEV), {n: i[n][0] for n in ("q", "k", "v", "delta")}
    i.update(flat, state=i["state"].expand(4, -1, -1, -1).contiguous())
    _check_forward(i, (3000,))


@pytest.mark.parametrize("strength", [0.0, 1e-3, 30.0, 1e4])
def test_decays_from_none_to_all(strength):
    lead = (2, 260)
    i = _inputs(lead, 2, 2, 2, 32, 32, B, 9, strength=strength)
    if strength == 0.0:
        i["A"].zero_()
    _check_forward(i, lead)


@pytest.mark.parametrize("dtype", [B, H])
def test_a_decay_of_minus_infinity_forgets_everything(dtype):
    lead = (1, 300)
    i = _inputs(lead, 1, 2, 1, 32, 64, dtype, 11, "head")
    i["delta"] = torch.zeros((*lead, 2), device=DEV, dtype=dtype)
    i["A"] = -torch.ones(2, device=DEV)
    for t in (0, 5, 6, 130, 200, 299):
        i["delta"][:, t, 1] = float("inf")
    _check_forward(i, lead)


def test_states_far_from_one_in_float16():
    """What queries meet is held in 16 bits: it is taken times a power of two."""
    lead = (1, 400)
    for a in (3e4, 1e-4):
        i = _inputs(lead, 1, 2, 2, 64, 96, H, 13, strength=1e-4)
        i["state"] *= a
        i["v"] = (i["v"].float() * min(a, 100.0)).to(H)
        i["q"] = (i["q"].float() * min(1.0, 1 / a)).to(H)
        lead_scale = 0.125
        _check_forward(i, lead, scale=lead_scale)


def test_large_products_in_float16():
    """The scale goes into the scores before they are rounded: q . k may pass the largest float16 as long as scale q . k does not."""
    lead = (1, 200)
    i = _inputs(lead, 1, 2, 2, 64, 64, H, 14, strength=0.01)
    i["q"], i["k"] = i["q"] * 100, i["k"] * 100                                     # q . k up to 4e5
    i["state"] *= 100
    _check_forward(i, lead, scale=1e-3)


def test_slices_of_wider_rows_and_state_in_place():
    g = torch.Generator(device=DEV).manual_seed(3)
    for pad in (0, 8, 3):                                                           # aligned to 16 bytes, or not
        wide = torch.randn((2, 140, 2 * 64 + 2 * 64 + 4 * 32 + 4 + pad), generator=g, device=DEV).to(B)
        q, k, v, delta = wide[..., :128].unflatten(-1, (2, 64)), wide[..., 128:256].unflatten(-1, (2, 64)), wide[..., 256:384].unflatten(-1, (4, 32)), wide[..., 384:388]
        i = dict(q=q, k=k, v=v, A=-torch.rand(4, generator=g, device=DEV), delta=delta, delta_bias=None, softplus=True, offsets=None,
                 state=torch.randn((2, 4, 64, 32), generator=g, device=DEV))
        args = _args(i, (2, 140), 0.125)
        want, last, _, _ = au.attend(*args)
        mag, mag_last, _, _ = au.attend(*args, magnitudes=True)
        rel, _ = _bounds(i, args, (2, 140))
        before = wide.clone()
        S = i["state"].clone()
        i["state"] = S
        y = _call(i, state_out=S, y=v if pad == 3 else None)                        # over v, and over the state
        au.within(y.reshape(want.shape), want, (au.half_step(B) + rel) * mag, B, "y")
        au.within(S, last, rel * mag_last, F, "state")
        if pad == 3:
            before[..., 256:384] = y.flatten(-2)
        assert torch.equal(wide, before)


@pytest.mark.parametrize("dk, dv", [(64, 64), (20, 33)])
def test_one_row_for_all_tokens_and_one_sequence_for_all(dk, dv):
    """Operands of stride zero, by expand: what their copies give."""
    i = _inputs((3, 150), 3, 4, 2, dk, dv, B, 15, grad=True)
    i["q"], i["v"], i["dy"] = i["q"][:, :1].expand(3, 150, 2, dk), i["v"][:1].expand(3, 150, 4, dv), i["dy"][:1, :1].expand(3, 150, 4, dv)
    call = lambda j: dict(block.decay_attention_grad(j["dy"], j["q"], j["k"], j["v"], j["A"], j["delta"], j["delta_bias"], True, None, j["state"], None, j["dlast"]), y=_call(j))  # noqa: E731
    got, want = call(i), call({n: t.contiguous() if torch.is_tensor(t) else t for n, t in i.items()})
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_tokens_of_all_sequences_beside_one_another_and_rows_over_one_another():
    """Strides in another order ([tokens, batch, ..]), and windows that overlap: what their copies give."""
    i = _inputs((3, 150), 3, 4, 2, 64, 64, B, 16, grad=True)
    for n in ("q", "v", "dy", "delta"):
        i[n] = i[n].transpose(0, 1).contiguous().transpose(0, 1)
    line = i["k"].flatten()
    i["k"] = line.as_strided((3, 150, 2, 64), (4096, 8, 64, 1))
    call = lambda j: dict(block.decay_attention_grad(j["dy"], j["q"], j["k"], j["v"], j["A"], j["delta"], j["delta_bias"], True, None, j["state"], None, j["dlast"]), y=_call(j))  # noqa: E731
    got, want = call(i), call({n: t.contiguous() if torch.is_tensor(t) else t for n, t in i.items()})
    assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("offsets", [None, [0, 1, 2000, 3000]])
def test_state_in_place_where_sequences_are_cut(offsets):
    """The first piece does not find what the last one leaves."""
    lead = (1, 3000) if offsets is None else (3000,)
    i = _inputs(lead, 1 if offsets is None else 3, 2, 1, 64, 64, B, 18, strength=0.01, offsets=offsets)
    last = torch.empty_like(i["state"])
    want, given = _call(i, state_out=last), i["state"].clone()
    for _ in range(20):
        i["state"].copy_(given)
        y = _call(i, state_out=i["state"])
        assert torch.equal(y, want) and torch.equal(i["state"], last)


def test_other_sequences_infinities_stay_there():
    i = _inputs((300,), 3, 2, 2, 64, 64, B, 17, offsets=[0, 100, 180, 300])
    clean = _call(i).clone()
    for n in ("q", "k", "v"):
        i[n][100:180] = float("nan")
        i[n][140] = float("inf")
    got = _call(i)
    assert torch.equal(got[:100], clean[:100]) and torch.equal(got[180:], clean[180:])


@pytest.mark.parametrize("dk, dv, dtype", [(64, 64, B), (128, 128, H), (36, 20, B), (7, 3, H), (100, 128, B)])
@pytest.mark.parametrize("decay", ["token", "head"])
def test_single_tokens(dk, dv, dtype, decay):
    i = _inputs((3,), 3, 4, 2, dk, dv, dtype, 19, decay)
    s = dk ** -0.5
    f = lambda n: au.f64(i[n])  # noqa: E731
    args = (f("q"), f("k"), f("v"), f("A"), f("delta"), f("delta_bias"), i["softplus"], s, f("state"), [(b, b + 1) for b in range(3)])
    want, last, _, _ = au.attend(*args)
    mag, mag_last, _, _ = au.attend(*args, magnitudes=True)
    S = i["state"].clone()
    y = block.decay_attention_step(i["q"], i["k"], i["v"], i["A"], S, i["delta"], i["delta_bias"], i["softplus"])
    R = dk + 8 * 200 + 16                                                           # exponents up to 200, one token: no 16-bit operands
    au.within(y, want, R * au.U * mag, dtype, "y")
    au.within(S, last, R * au.U * mag_last, F, "state")


def test_a_prompt_is_its_tokens_one_by_one():
    lead = (2, 40)
    i = _inputs(lead, 2, 3, 1, 48, 64, B, 23)
    S = i["state"].clone()
    steps = [block.decay_attention_step(i["q"][:, t], i["k"][:, t], i["v"][:, t], i["A"], S, i["delta"][:, t], i["delta_bias"], True) for t in range(40)]
    last = torch.empty_like(S)
    y = _call(i, state_out=last)
    args = _args(i, lead, 48 ** -0.5)
    mag, mag_last, _, _ = au.attend(*args, magnitudes=True)
    rel, _ = _bounds(i, args, lead)
    h = au.half_step(B)
    off = np.abs(au.f64(y) - au.f64(torch.stack(steps, 1))).reshape(mag.shape)
    assert (off <= (3 * h + 2 * rel) * mag).all()                                   # scores or states, and both results rounded
    assert (np.abs(au.f64(last) - au.f64(S)) <= 2 * rel * mag_last).all()


# ---- gradients ------------------------------------------------------------------------------------------------------------

def _check_gradients(i, lead, scale=None, want=None, **kw):
    s = i["q"].shape[-1] ** -0.5 if scale is None else scale
    args = _args(i, lead, s)
    dy, dlast = _flat(i["dy"], lead), au.f64(i["dlast"])
    ref = au.attend_grad(dy, *args, dlast)
    mag = au.attend_grad(dy, *args, dlast, magnitudes=True)
    rel, chunks = _bounds(i, args, lead)
    got = block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], i["softplus"], scale, i["state"], i["offsets"], i["dlast"],
                                     want=want, **kw)
    assert set(got) == set(want or ref)
    inside = np.zeros(dy.shape[0], bool)
    for lo, hi in args[-1]:
        inside[lo:hi] = True
    at = torch.from_numpy(inside).to(DEV)
    h = au.half_step(i["q"].dtype)
    for n in got:
        if n in ("dq", "dk", "dv", "ddelta"):
            t = got[n].reshape(ref[n].shape)[at]
            au.within(t, ref[n][inside], ((0 if n == "ddelta" else h) + 2 * rel + 256 * au.U) * mag[n][inside], got[n].dtype, n)
        else:
            au.within(got[n], ref[n], (2 * rel + (256 + dy.shape[0]) * au.U) * mag[n], F, n)
    assert block.device_error(0) == 0
    return got


@pytest.mark.parametrize("tokens", [1, 31, 33, 128, 129, 390])
@pytest.mark.parametrize("dk, dv, dtype", [(64, 64, B), (128, 128, B), (128, 64, H), (64, 128, H), (128, 128, H)])
def test_gradients_lengths(tokens, dk, dv, dtype):
    lead = (2, tokens)
    _check_gradients(_inputs(lead, 2, 2, 2, dk, dv, dtype, tokens + 1, grad=True), lead)


@pytest.mark.parametrize("heads, groups, dk, dv, decay", [(6, 2, 36, 20, "token"), (4, 1, 7, 66, "token"), (3, 3, 72, 8, "head"), (4, 1, 128, 64, "head"), (8, 4, 64, 64, "token")])
@pytest.mark.parametrize("dtype", [B, H])
def test_gradients_of_shared_heads_and_odd_widths(heads, groups, dk, dv, decay, dtype):
    lead = (2, 140)
    _check_gradients(_inputs(lead, 2, heads, groups, dk, dv, dtype, dk, decay, grad=True), lead, scale=0.3)


@pytest.mark.parametrize("offsets, rows", [([0, 0, 130, 130, 131, 400], 400), ([3, 60, 60, 64, 199], 210), ([0, 1, 2], 2)])
@pytest.mark.parametrize("dk, dtype, groups", [(64, B, 2), (40, H, 4)])
def test_gradients_of_packed_sequences(offsets, rows, dk, dtype, groups):
    _check_gradients(_inputs((rows,), len(offsets) - 1, 4, groups, dk, 64, dtype, rows, offsets=offsets, grad=True), (rows,))


def test_gradients_of_a_long_sequence_in_pieces_and_of_none():
    _check_gradients(_inputs((1, 1500), 1, 1, 1, 64, 32, B, 29, strength=0.05, grad=True), (1, 1500))
    got = block.decay_attention_grad(*(torch.zeros((0, 2, 8), device=DEV, dtype=B) for _ in range(4)), -torch.ones(2, device=DEV),
                                     offsets=torch.zeros(3, dtype=torch.int32, device=DEV), dstate_out=torch.ones((2, 2, 8, 8), device=DEV))
    assert bool((got["dA"] == 0).all()) and bool((got["dstate"] == 1).all())


def test_gradients_without_states_some_wanted_and_outputs_handed_in():
    lead = (1, 200)
    i = _inputs(lead, 1, 2, 2, 64, 64, B, 31, state=False, grad=True)
    every = _check_gradients(i, lead)
    for want in (["dq"], ["dk"], ["dv", "dstate"], ["dA"], ["ddelta"], ["dq", "dk", "dv"]):
        some = _check_gradients(i, lead, want=want, out={n: torch.full_like(every[n], float("nan")) for n in want})
        for n in want:
            if n in ("dstate", "dA", "ddelta"):                                     # (dq, dk, dv alone make do with states in two terms)
                assert torch.equal(some[n], every[n]), n


def test_gradients_with_strong_and_infinite_decays():
    lead = (1, 260)
    for strength in (0.0, 1e-3, 50.0):
        i = _inputs(lead, 1, 2, 2, 32, 32, B, 37, strength=strength, grad=True)
        if strength == 0.0:
            i["A"].zero_()
        _check_gradients(i, lead)


@pytest.mark.parametrize("softplus", [True, False])
def test_steps_of_infinity_and_decays_of_minus_infinity(softplus):
    """A step of infinity forgets as any other does whose decay is zero in float32, and has no share in the gradients of A and delta; a decay of minus
    infinity forgets everything, but keeps the state over a step of nothing (of zero, or a softplus below the numbers there are)."""
    lead = (1, 200)
    i = _inputs(lead, 1, 3, 1, 32, 40, B, 39, grad=True)
    i["softplus"], i["delta_bias"], i["delta"] = softplus, None, i["delta"].abs()
    i["A"] = torch.tensor([-1.0, -0.5, -1.0], device=DEV)

    def all_of():
        last, S = torch.empty_like(i["state"]), i["state"].clone()
        got = block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], None, softplus, None, i["state"], None, i["dlast"])
        got.update(y=_call(i, state_out=last), last=last)
        got["one"] = block.decay_attention_step(i["q"][:, 5], i["k"][:, 5], i["v"][:, 5], i["A"], S, i["delta"][:, 5], None, softplus)
        got["S"] = S
        return got

    i["delta"][:, 0::3, 2], i["delta"][:, 1::3, 2] = 1.0, 2.0
    i["delta"][:, 2::3, 2] = -200.0 if softplus else 0.0                            # a step of nothing
    results = []
    for large, lowest in ((1e4, -1e4), (float("inf"), float("-inf"))):
        for t in (0, 5, 6, 130, 199):
            i["delta"][:, t, 1] = large
        i["A"][2] = lowest
        results.append(all_of())
    for n in results[0]:
        one, two = results[0][n], results[1][n]
        if n in ("ddelta", "ddelta_bias"):                                          # (A times what passes through a decay: not finite where A is not)
            one, two = one[..., :2], two[..., :2]
        assert torch.isfinite(two).all(), n
        assert torch.equal(one, two), n


def test_the_same_call_gives_the_same_bits():
    i = _inputs((2, 300), 2, 4, 2, 64, 64, H, 41, grad=True)
    call = lambda: block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], True, None, i["state"], None, i["dlast"])  # noqa: E731
    one, two = call(), call()
    assert all(torch.equal(one[n], two[n]) for n in one)
    assert torch.equal(_call(i), _call(i))


@pytest.mark.parametrize("dk, dv, dtype, rows, offsets", [(40, 64, H, 400, [0, 0, 130, 130, 131, 400]), (7, 66, H, 140, [0, 140]), (100, 30, B, 600, [0, 600]), (64, 64, H, 700, [0, 700])])
def test_what_scratch_held_before_does_not_matter(dk, dv, dtype, rows, offsets):
    i = _inputs((rows,), len(offsets) - 1, 2, 1, dk, dv, dtype, 47, offsets=offsets, grad=True)

    def both():
        last = torch.empty_like(i["state"])
        got = block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], True, None, i["state"], i["offsets"], i["dlast"])
        return dict(got, y=_call(i, state_out=last), last=last)

    first = both()
    for fill in (0, 255, 0x7e):
        for size in (1 << 16, 1 << 20, 1 << 24, 1 << 26):                           # of all sizes that the allocator keeps apart
            torch.full((size,), fill, dtype=torch.uint8, device=DEV)
        got = both()
        assert all(torch.equal(got[n], first[n]) for n in first), fill


# ---- streams, graphs, many calls ------------------------------------------------------------------------------------------

def test_another_stream_and_a_captured_call():
    i = _inputs((2, 300), 2, 4, 2, 64, 64, B, 43, grad=True)
    want, last = torch.empty_like(i["v"]), torch.empty_like(i["state"])
    _call(i, y=want, state_out=last)
    grads = block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], True, None, i["state"])
    s = torch.cuda.Stream(device=DEV)
    torch.cuda.synchronize()
    y = _call(i, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    S = i["state"].clone()
    with torch.cuda.graph(g):
        y = _call(i)
        got = block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], True, None, i["state"])
        one = block.decay_attention_step(i["q"][:, 0], i["k"][:, 0], i["v"][:, 0], i["A"], S, i["delta"][:, 0], i["delta_bias"], True)
    y.zero_()
    for _ in range(3):
        S.copy_(i["state"])
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and all(torch.equal(got[n], grads[n]) for n in got)
    S.copy_(i["state"])
    assert torch.equal(one, block.decay_attention_step(i["q"][:, 0], i["k"][:, 0], i["v"][:, 0], i["A"], S, i["delta"][:, 0], i["delta_bias"], True))


def test_many_calls_one_behind_another():
    """Waits of one call do not see signals of another: four hundred of them, of different sizes."""
    some = [_inputs((b, n), b, h, h, dk, 64, B, n) for b, n, h, dk in ((1, 1500, 4, 64), (4, 513, 8, 128), (2, 100, 2, 64))]
    want = [_call(i).clone() for i in some]
    for _ in range(130):
        got = [_call(i) for i in some]
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and block.device_error(0) == 0


def test_two_streams_at_once():
    some = [_inputs((2, 700), 2, 8, 4, 64, 64, B, n, grad=True) for n in (1, 2)]
    grads = lambda i, **kw: block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], True, None, i["state"], None, i["dlast"], **kw)  # noqa: E731
    want = [(_call(i), grads(i)) for i in some]
    streams = [torch.cuda.Stream(device=DEV) for _ in some]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for i, s in zip(some, streams):
            with torch.cuda.stream(s):
                got.append((_call(i), grads(i)))
    torch.cuda.synchronize()
    for n, (y, g) in enumerate(got):
        assert torch.equal(y, want[n % 2][0]) and all(torch.equal(g[m], want[n % 2][1][m]) for m in g)


def test_two_captured_calls_replayed_in_turn():
    """Each graph has its own scratch: neither finds what the other left wrong."""
    some = [_inputs((1, n), 1, 2, 1, 64, 64, B, n, grad=True) for n in (1500, 900)]  # cut into pieces: states in scratch
    grads = lambda i: block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], True, None, i["state"], None, i["dlast"])  # noqa: E731
    want = [(_call(i).clone(), {n: t.clone() for n, t in grads(i).items()}) for i in some]
    graphs, got = [torch.cuda.CUDAGraph() for _ in some], []
    torch.cuda.synchronize()
    for g, i in zip(graphs, some):
        with torch.cuda.graph(g):
            got.append((_call(i), grads(i)))
    for n in (0, 1, 1, 0, 1, 0):
        graphs[n].replay()
        assert torch.equal(got[n][0], want[n][0]) and all(torch.equal(got[n][1][m], want[n][1][m]) for m in want[n][1])


def test_rows_past_32_bits():
    """Rows of 2.4e9 elements in all: operands and results are slices of them."""
    tokens, heads, d = 60000, 2, 64
    g = torch.Generator(device=DEV).manual_seed(3)
    wide = torch.zeros((tokens, 40000), device=DEV, dtype=B)
    slices = [wide[:, at:at + heads * d].unflatten(-1, (heads, d)) for at in (0, 8000, 16000, 24000, 32000)]
    q, k, v, dy, y = slices
    for t in (q, k, v, dy):
        t.copy_(torch.randn(t.shape, generator=g, device=DEV))
    A = torch.tensor([-0.01, -0.2], device=DEV)
    offsets = torch.tensor([0, 100, 59000, 59990], dtype=torch.int32, device=DEV)
    c = lambda t: t.contiguous()  # noqa: E731
    want = block.decay_attention(c(q), c(k), c(v), A, offsets=offsets, y=torch.zeros_like(c(v)))
    block.decay_attention(q, k, v, A, offsets=offsets, y=y)
    assert torch.equal(y, want) and bool((y[59990:] == 0).all()) and bool(y[59000:59990].any())
    some = ["dq", "dk", "dv"]
    new = lambda: {n: torch.zeros((tokens, heads, d), device=DEV, dtype=B) for n in some}  # noqa: E731
    want = block.decay_attention_grad(c(dy), c(q), c(k), c(v), A, offsets=offsets, want=some, out=new())
    got = block.decay_attention_grad(dy, q, k, v, A, offsets=offsets, want=some, out=new())
    assert all(torch.equal(got[n], want[n]) and bool(got[n][59000:59990].any()) for n in some)


def test_no_tokens_and_no_sequences():
    g = torch.Generator(device=DEV).manual_seed(5)
    S, A = torch.randn((2, 3, 16, 24), generator=g, device=DEV), -torch.ones(3, device=DEV)
    q, v = torch.zeros((2, 0, 1, 16), device=DEV, dtype=B), torch.zeros((2, 0, 3, 24), device=DEV, dtype=B)
    last = torch.full_like(S, float("nan"))
    assert block.decay_attention(q, q, v, A, state=S, state_out=last).shape == v.shape
    got = block.decay_attention_grad(v, q, q, v, A, state=S, dstate_out=2 * S)
    assert torch.equal(last, S) and torch.equal(got["dstate"], 2 * S) and bool((got["dA"] == 0).all()) and got["dq"].shape == q.shape
    none = block.decay_attention(q[:0], q[:0], v[:0], A)
    assert none.shape == (0, 0, 3, 24)
    one = block.decay_attention_step(q[:0, 0:0].reshape(0, 1, 16), q[:0].reshape(0, 1, 16), v[:0].reshape(0, 3, 24), A, S[:0])
    assert one.shape == (0, 3, 24)


def test_calls_from_several_threads():
    import threading

    some = [_inputs((2, n), 2, 4, 2, 64, 64, B, n, grad=True) for n in (200, 300, 500, 1400)]
    both = lambda i: (_call(i), block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], True, None, i["state"])["dk"],  # noqa: E731
                      block.block_norm(i["v"].flatten(-2), w_pre=torch.ones(256, device=DEV))[1])
    want, wrong = [both(i) for i in some], []
    torch.cuda.synchronize()

    def work(i, w):
        s = torch.cuda.Stream(device=DEV)
        with torch.cuda.stream(s):
            for _ in range(20):
                got = both(i)
                s.synchronize()
                wrong.extend(n for n in range(3) if not torch.equal(got[n], w[n]))

    threads = [threading.Thread(target=work, args=a) for a in zip(some, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and block.device_error(0) == 0


@pytest.mark.parametrize("dtype", [B, H])
@pytest.mark.parametrize("heads, offsets", [(2, [-50, 200, 100, 1 << 30, 250]), (2, [0, 300] * 10 + [0]), (40, [0, 300] * 10 + [0]), (2, [0, 300] * 40)])
def test_offsets_that_make_no_sense_stay_in_range(monkeypatch, heads, offsets, dtype):
    """Offsets beyond the rows and ones that jump back, which ask for more chunks than there is room for: nothing outside of scratch and results is touched."""
    kept = []

    def guarded(need, x, stream):
        block._check(min(need, 0))
        kept.append((torch.full((need + 512,), 0x5a, dtype=torch.uint8, device=DEV), need))
        return kept[-1][0], kept[-1][0].data_ptr() + 256

    monkeypatch.setattr(block, "_workspace", guarded)
    block._load()
    monkeypatch.setattr(block, "_step", block._LongWay)                           # (the short way has scratch of its own)
    i = _inputs((300,), len(offsets) - 1, heads, heads, 64, 64, dtype, 51, offsets=offsets, grad=True)
    guard = torch.full((500, heads, 64), 3.0, device=DEV, dtype=dtype)
    last = torch.empty_like(i["state"])
    _call(i, y=guard[100:400], state_out=last)
    block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], i["delta_bias"], True, None, i["state"], i["offsets"], i["dlast"])
    torch.cuda.synchronize()
    assert len(kept) == 2 and bool((guard[:100] == 3).all()) and bool((guard[400:] == 3).all()) and block.device_error(0) == 0
    for ws, need in kept:
        assert bool((ws[:256] == 0x5a).all()) and bool((ws[256 + need:] == 0x5a).all())
