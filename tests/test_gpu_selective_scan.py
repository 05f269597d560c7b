"""Selective scan, its gradients and its step against the plain 64-bit form (bounds: block_util.py)."""
import numpy as np
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import block_util as bu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = torch.float32
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _inputs(batch, lead, d, n, dtype, groups=1, gated=True, skip=True, bias=True, state=True, softplus=True, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s, t=dtype: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    delta = r(*lead, d) if softplus else r(*lead, d).abs() * 0.3
    return dict(x=r(*lead, d), delta=delta, A=-torch.rand((d, n), generator=g, device=DEV) * 2 - 0.05, B=r(*lead, groups, n), C=r(*lead, groups, n),
                D=r(d, t=F) if skip else None, z=r(*lead, d) if gated else None, delta_bias=r(d, t=F) * 0.5 - 1 if bias and softplus else None,
                softplus=softplus, state=r(batch, d, n, t=F) if state else None)


def _plain(v, lead, offsets):
    flat = lambda t, k: None if t is None else bu.f64(t).reshape(-1, *t.shape[len(lead):])  # noqa: E731
    a = {k: flat(v[k], k) for k in ("x", "delta", "B", "C", "z")}
    if a["B"].ndim == 2:
        a["B"], a["C"] = a["B"][:, None], a["C"][:, None]
    return dict(a, A=bu.f64(v["A"]), D=bu.f64(v["D"]), delta_bias=bu.f64(v["delta_bias"]), softplus=v["softplus"], state=bu.f64(v["state"]),
                seqs=bu.spans(lead, offsets))


def _roundings(a):
    step, _ = bu.scan_step_sizes(a["delta"], a["delta_bias"], a["softplus"])
    largest = np.abs(step).max(initial=0.0) * np.abs(a["A"]).max()
    longest = max([hi - lo for lo, hi in a["seqs"]] + [0])
    return bu.scan_roundings(longest, a["x"].shape[0], a["x"].shape[1], a["A"].shape[1], largest)


def _inside(want):
    return ~np.isnan(want).reshape(want.shape[0], -1).any(1)


def _check_rows(got, want, bound, dtype, what):
    keep = _inside(want)
    got = got.reshape(want.shape)[torch.from_numpy(keep).to(DEV)]
    bu.within(got, want[keep], bound[keep], dtype, what)


def _check_forward(v, lead, offsets=None, y=None, state_out="new"):
    a = _plain(v, lead, offsets)
    batch, (d, n) = len(a["seqs"]), a["A"].shape
    last = v["state"] if state_out == "same" else torch.full((batch, d, n), 7.0, device=DEV)
    got = block.selective_scan(**v, offsets=offsets, y=y, state_out=last)
    want, states, _ = bu.scan(**a)
    mag, state_mag, _ = bu.scan(**a, magnitudes=True)
    r = _roundings(a) * bu.U
    _check_rows(got, want, r * mag, v["x"].dtype, "y")
    bu.within(last, states, r * state_mag, F, "state_out")
    return got, last


def _check_grad(v, lead, offsets=None, dlast=True, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    a = _plain(v, lead, offsets)
    dy = torch.randn(v["x"].shape, generator=g, device=DEV).to(v["x"].dtype)
    dlast = torch.randn((len(a["seqs"]), *a["A"].shape), generator=g, device=DEV) if dlast else None
    got = block.selective_scan_grad(dy, **v, offsets=offsets, dstate_out=dlast)
    more = dict(a, dy=bu.f64(dy).reshape(a["x"].shape), dlast=bu.f64(dlast))
    want, mag = bu.scan_grad(**more), bu.scan_grad(**more, magnitudes=True)
    assert set(got) == set(want)
    r = 2 * _roundings(a) * bu.U                                     # a product may hold a state and a co-state
    for k in want:
        if k in ("dx", "ddelta", "dz", "dB", "dC"):
            _check_rows(got[k], want[k], r * mag[k], v["x"].dtype, k)
        else:
            bu.within(got[k], want[k], r * mag[k], F, k)
    return dy, got


SHAPES = [(1, 1, 1, 1, 1), (2, 2, 5, 3, 1), (1, 15, 32, 4, 1), (3, 16, 33, 16, 1), (2, 17, 8, 5, 2), (1, 70, 24, 24, 3), (2, 33, 12, 64, 1),
          (1, 40, 10, 100, 2), (1, 65, 7, 128, 1), (2, 64, 130, 8, 1), (1, 129, 40, 16, 4)]                    # batch, tokens, d, n, groups


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_equal_sequences(shape, dtype):
    batch, tokens, d, n, groups = shape
    v = _inputs(batch, (batch, tokens), d, n, dtype, groups)
    _check_forward(v, (batch, tokens))
    _check_grad(v, (batch, tokens))


@pytest.mark.parametrize("option", ["gated", "skip", "bias", "state", "softplus"])
def test_without(option):
    v = _inputs(2, (2, 37), 20, 16, F, groups=2, **{option: False})
    _check_forward(v, (2, 37))
    _check_grad(v, (2, 37))
    _check_grad(v, (2, 37), dlast=False)
    v["B"], v["C"] = v["B"][:, :, 0].contiguous(), v["C"][:, :, 0].contiguous()                              # one group without its axis
    _check_forward(v, (2, 37))
    dy, g = _check_grad(v, (2, 37))
    assert g["dB"].shape == v["B"].shape


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cuts, rows", [([0, 0, 1, 4, 4, 80, 113, 113], 113), ([3, 40, 41, 43], 50), ([0, 0], 5), ([2, 2, 2], 4), ([0, 64, 128, 192], 192)])
def test_packed_sequences_and_rows_outside_of_them(cuts, rows, dtype):
    offsets = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    v = _inputs(len(cuts) - 1, (rows,), 24, 16, dtype, groups=2)
    y = torch.full_like(v["x"], 99.0)
    _check_forward(v, (rows,), offsets, y=y)
    assert bool((y[:cuts[0]] == 99).all()) and bool((y[cuts[-1]:] == 99).all())
    _check_grad(v, (rows,), offsets)
    out = {k: torch.full_like(v[k[1:]], 99.0) for k in ("dx", "ddelta", "dz", "dB", "dC")}
    block.selective_scan_grad(v["x"], **v, offsets=offsets, want=tuple(out), out=out)
    for t in out.values():
        assert bool((t[:cuts[0]] == 99).all()) and bool((t[cuts[-1]:] == 99).all())


# Few channels and many tokens: cut into pieces of tokens.
@pytest.mark.parametrize("batch, tokens, d, n", [(1, 1025, 8, 16), (2, 700, 3, 4), (1, 513, 40, 64), (1, 256, 16, 2)])
def test_long_sequences_of_few_channels(batch, tokens, d, n):
    v = _inputs(batch, (batch, tokens), d, n, F)
    _check_forward(v, (batch, tokens))
    _check_grad(v, (batch, tokens))
    v["state"] = None
    _check_forward(v, (batch, tokens))


def test_long_packed_sequences_of_few_channels():
    cuts = [0, 0, 5, 400, 400, 1300, 1301, 1301]
    offsets = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    v = _inputs(len(cuts) - 1, (1310,), 8, 16, torch.bfloat16)
    y = torch.full_like(v["x"], 99.0)
    _check_forward(v, (1310,), offsets, y=y)
    assert bool((y[1301:] == 99).all())
    _check_grad(v, (1310,), offsets)


@pytest.mark.parametrize("lead, cuts", [((2, 700), None), ((2, 40), None), ((1000,), [0, 300, 300, 1000])])
def test_state_in_place_and_output_over_inputs(lead, cuts):
    offsets = None if cuts is None else torch.tensor(cuts, dtype=torch.int32, device=DEV)
    batch = lead[0] if cuts is None else len(cuts) - 1
    v = _inputs(batch, lead, 6, 16, F)
    y, last = block.selective_scan(**v, offsets=offsets, state_out=(s := torch.empty_like(v["state"]))), s
    for over in ("x", "z"):
        u = {k: t.clone() if torch.is_tensor(t) else t for k, t in v.items()}
        got = block.selective_scan(**u, offsets=offsets, y=u[over], state_out=u["state"])
        assert torch.equal(got, y) and torch.equal(u["state"], last)


@pytest.mark.parametrize("tokens", [1, 16, 33, 128])
def test_a_prompt_in_two_calls(tokens):
    v = _inputs(2, (2, 150), 12, 16, F)
    a = _plain(v, (2, 150), None)
    want, states, _ = bu.scan(**a)
    mag, state_mag, _ = bu.scan(**a, magnitudes=True)
    state = v["state"].clone()
    rows = ("x", "delta", "B", "C", "z")
    ys = []
    for part in (slice(0, tokens), slice(tokens, 150)):
        ys.append(block.selective_scan(**{**v, **{k: v[k][:, part] for k in rows}, "state": state}, state_out=state))
    r = _roundings(a) * bu.U
    _check_rows(torch.cat(ys, 1), want, r * mag, F, "y")
    bu.within(state, states, r * state_mag, F, "state")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch, d, n, groups", [(1, 1, 1, 1), (3, 33, 16, 1), (2, 64, 16, 4), (5, 6, 7, 2), (2, 9, 128, 1), (150, 40, 4, 1)])
def test_step_against_the_plain_form(batch, d, n, groups, dtype):
    v = _inputs(batch, (batch, 3), d, n, dtype, groups)
    a = _plain(v, (batch, 3), None)
    want, states, _ = bu.scan(**a)
    mag, state_mag, _ = bu.scan(**a, magnitudes=True)
    r = _roundings(a) * bu.U
    state = v.pop("state").clone()
    ys = [block.selective_scan_step(**{**v, **{k: v[k][:, t] for k in ("x", "delta", "B", "C", "z")}}, state=state) for t in range(3)]
    _check_rows(torch.stack(ys, 1), want, r * mag, dtype, "y")
    bu.within(state, states, r * state_mag, F, "state")


@pytest.mark.parametrize("off", [0, 1, 3])
def test_slices_of_wider_rows_and_states_off_16_bytes(off):
    d, n = 20, 16
    v = _inputs(2, (2, 45), d, n, torch.bfloat16)
    wide = torch.randn((2, 45, 3 * d + 2 * n + 8), device=DEV).bfloat16()
    at = off
    for k, w in (("x", d), ("delta", d), ("z", d)):
        v[k], at = wide[..., at:at + w], at + w
    v["B"], v["C"] = wide[..., at:at + n], wide[..., at + n:at + 2 * n]
    _check_forward(v, (2, 45))
    _check_grad(v, (2, 45))
    room = torch.randn(2 * d * n + 1, device=DEV)
    state = room[1:].view(2, d, n)
    step = {**v, **{k: v[k][:, 0] for k in ("x", "delta", "B", "C", "z")}, "state": state.clone()}
    y = block.selective_scan_step(**step)
    step2 = {**step, "state": state}
    assert torch.equal(block.selective_scan_step(**step2), y) and torch.equal(state, step["state"])


def test_no_sequences_and_no_tokens():
    v = _inputs(0, (0, 5), 8, 4, torch.bfloat16)
    assert block.selective_scan(**v).shape == (0, 5, 8)
    g = block.selective_scan_grad(v["x"], **v)
    assert not g["dA"].any() and not g["dD"].any() and not g["ddelta_bias"].any()
    v = _inputs(2, (2, 0), 8, 4, torch.bfloat16)
    last = torch.empty_like(v["state"])
    block.selective_scan(**v, state_out=last)
    assert torch.equal(last, v["state"])
    g = block.selective_scan_grad(v["x"], **v, dstate_out=v["state"])
    assert torch.equal(g["dstate"], v["state"]) and not g["dA"].any()


def test_extreme_step_sizes():
    """Decays that underflow to nothing, steps of nothing, and softplus far from zero on both sides."""
    v = _inputs(1, (1, 40), 8, 16, F)
    v["delta"][0, ::3] = 90.0
    v["delta"][0, 1::3] = -200.0
    v["A"][:] = -torch.arange(1, 17, device=DEV) * 10.0
    y = block.selective_scan(**v)
    a = _plain(v, (1, 40), None)
    want, _, _ = bu.scan(**a)
    mag, _, _ = bu.scan(**a, magnitudes=True)
    assert torch.isfinite(y).all()
    # a step of 90 leaves exp(-900); a step of exp(-200) is below float32 and is nothing: 24 operations on what is left
    bu.within(y.reshape(40, 8), want, (24 + 16) * 4 * bu.U * mag, F, "y")
    g = block.selective_scan_grad(torch.ones_like(y), **v)
    assert all(torch.isfinite(t).all() for t in g.values())


def test_nan_stays_in_its_channel():
    v = _inputs(1, (1, 50), 40, 16, F)
    v["x"][0, 20, 7] = float("nan")
    y = block.selective_scan(**v)
    bad = torch.isnan(y[0])
    assert bad[20:, 7].all() and int(bad.sum()) == 30
    v["x"][0, 20, 7] = float("inf")
    y = block.selective_scan(**v)
    assert torch.isfinite(y[0][:, :7]).all() and torch.isfinite(y[0][:20]).all()


def test_offsets_that_make_no_sense_stay_in_range():
    """Offsets beyond the rows and decreasing ones: clamped, nothing outside the tensors is touched."""
    v = _inputs(4, (300,), 8, 16, F)
    offsets = torch.tensor([-50, 200, 100, 1 << 30, 250], dtype=torch.int32, device=DEV)
    guard = torch.full((500, 8), 3.0, device=DEV)
    block.selective_scan(**v, offsets=offsets, y=guard[100:400])
    block.selective_scan_grad(v["x"], **v, offsets=offsets)
    block.causal_conv(v["x"], torch.ones(8, 4, device=DEV), offsets=offsets, y=torch.empty_like(v["x"]), state_out=torch.empty(4, 3, 8, device=DEV))
    torch.cuda.synchronize()
    assert bool((guard[:100] == 3).all()) and bool((guard[400:] == 3).all())


@pytest.mark.parametrize("d, n", [(4, 4), (300, 16)])
def test_many_short_sequences(d, n):
    lengths = torch.randint(0, 4, (3000,), generator=torch.Generator().manual_seed(5))
    cuts = [0, *lengths.cumsum(0).tolist()]
    offsets = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    v = _inputs(len(cuts) - 1, (cuts[-1],), d, n, F)
    _check_forward(v, (cuts[-1],), offsets)
    if d == 4:
        _check_grad(v, (cuts[-1],), offsets)


def test_a_decay_of_minus_infinity():
    """exp(D A) = 0: the state is the last token's share, at tokens that do not fill a tile too."""
    v = _inputs(1, (1, 21), 6, 16, F)
    v["A"][2] = float("-inf")
    last = torch.empty((1, 6, 16), device=DEV)
    y = block.selective_scan(**v, state_out=last)
    assert torch.isfinite(y).all() and torch.isfinite(last).all()
    step = torch.nn.functional.softplus(v["delta"][0, -1, 2].double() + v["delta_bias"][2].double())
    want = float(step * v["x"][0, -1, 2].double()) * v["B"][0, -1, 0].double()
    bu.within(last[0, 2], bu.f64(want), 24 * bu.U * np.abs(bu.f64(want)), F, "state")


def test_the_same_bits_again_and_in_captured_graphs():
    v = _inputs(2, (2, 500), 24, 16, torch.bfloat16)
    dy = torch.randn((2, 500, 24), device=DEV).bfloat16()
    first, y = block.selective_scan_grad(dy, **v), block.selective_scan(**v)
    graphs, kept = [], []
    for _ in range(2):                                               # two graphs, each with its own scratch
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept.append((block.selective_scan_grad(dy, **v), block.selective_scan(**v)))
        graphs.append(graph)
    side = torch.cuda.Stream()
    for _ in range(3):                                               # side by side on two streams
        side.wait_stream(torch.cuda.current_stream())
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for g, again in kept:
            assert torch.equal(again, y)
            for k in first:
                assert torch.equal(first[k], g[k]), k
