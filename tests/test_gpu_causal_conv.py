"""Causal convolution, its gradients and its step against the plain 64-bit form (bounds: block_util.py)."""
import numpy as np
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import block_util as bu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = torch.float32
TYPES = [torch.bfloat16, torch.float16, torch.float32]
SHAPES = [(1, 1, 1, 4), (3, 2, 5, 4), (2, 17, 96, 4), (1, 300, 8, 3), (2, 130, 33, 2), (5, 3, 264, 4)]     # batch, tokens, d, taps


def _inputs(batch, lead, d, taps, dtype, seed=0, window=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s, t=dtype: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    return dict(x=r(*lead, d), w=r(d, taps, t=F) * taps ** -0.5, bias=r(d, t=F), state=r(batch, taps - 1, d) if window else None)


def _plain(v, act, lead, offsets):
    flat = lambda t: bu.f64(t).reshape(-1, t.shape[-1])  # noqa: E731
    return flat(v["x"]), bu.f64(v["w"]), None if v["bias"] is None else bu.f64(v["bias"]), act, bu.f64(v["state"]), bu.spans(lead, offsets)


def _forward_bound(args, z, act):
    x, w, bias, _, state, seqs = args
    mag = bu.conv(np.abs(x), np.abs(w), None if bias is None else np.abs(bias), "none", None if state is None else np.abs(state), seqs)[0]
    e = (w.shape[1] + 1) * bu.U * mag                                # of z: one rounding for each tap
    # the activation's slope is at most 1.1; exp, a sum, a division and a product: 8 u of the result
    return 1.1 * e + 8 * bu.U * np.abs(z) if act == "silu" else e


def _check_forward(v, act, lead, offsets=None, y=None, state_out="new"):
    last = torch.full_like(v["state"], 7.0) if state_out == "new" and v["state"] is not None else v["state"] if state_out == "same" else None
    args = _plain(v, act, lead, offsets)
    got = block.causal_conv(v["x"], v["w"], v["bias"], act=act, state=v["state"], offsets=offsets, y=y, state_out=last)
    want, windows, z = bu.conv(*args)
    bound = _forward_bound(args, z, act)
    inside = ~np.isnan(want).any(1)
    flat = got.reshape(-1, got.shape[-1])[torch.from_numpy(inside).to(DEV)]
    bu.within(flat, want[inside], bound[inside], got.dtype, "y")
    if last is not None:
        assert np.array_equal(bu.f64(last), windows)
    return got


def _check_grad(v, act, lead, offsets=None, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dy = torch.randn(v["x"].shape, generator=g, device=DEV).to(v["x"].dtype)
    args = _plain(v, act, lead, offsets)
    batch = len(args[-1])
    dlast = torch.randn((batch, v["w"].shape[1] - 1, v["w"].shape[0]), generator=g, device=DEV).to(v["x"].dtype)
    got = block.causal_conv_grad(dy, v["x"], v["w"], v["bias"], act=act, state=v["state"], offsets=offsets, dstate_out=dlast)
    more = (bu.f64(dy).reshape(-1, dy.shape[-1]), *args, bu.f64(dlast))
    want, mag = bu.conv_grad(*more), bu.conv_grad(*more, magnitudes=True)
    # z's error moves the slope (second derivative at most 0.5 in magnitude): by at most 0.5 (taps + 1) u |z|-magnitudes, which
    # the slope's share of the count stands for where they are below 16; longest path: rows for dw and dbias, taps for dx
    rows, taps = args[0].shape[0], v["w"].shape[1]
    x, w, bias, _, state, seqs = args
    zmag = bu.conv(np.abs(x), np.abs(w), None if bias is None else np.abs(bias), "none", None if state is None else np.abs(state), seqs)[0]
    dz_extra = 0.5 * (taps + 1) * bu.U * np.nanmax(zmag, initial=0.0) if act == "silu" else 0.0
    unit = bu.conv_grad(more[0], *args[:3], "none", *args[4:], None, magnitudes=True)       # dz's error through the sums
    for k, r in (("dx", taps + 20), ("dstate", taps + 20), ("dw", rows + 20), ("dbias", rows + 20)):
        bound = r * bu.U * mag[k] + dz_extra * unit[k]
        have = got[k].reshape(want[k].shape)
        if k == "dx":
            inside = ~np.isnan(want[k]).any(1)
            have, want[k], bound = have[torch.from_numpy(inside).to(DEV)], want[k][inside], bound[inside]
        bu.within(have, want[k], bound, v["x"].dtype if k in ("dx", "dstate") else F, k)
    return dy, got


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_equal_sequences(shape, dtype, act):
    batch, tokens, d, taps = shape
    v = _inputs(batch, (batch, tokens), d, taps, dtype)
    _check_forward(v, act, (batch, tokens))
    _check_grad(v, act, (batch, tokens))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cuts, rows", [([0, 0, 1, 4, 4, 150, 163, 163], 163), ([3, 40, 41, 43], 50), ([0, 0], 5), ([2, 2, 2], 4)])
def test_packed_sequences_and_rows_outside_of_them(cuts, rows, dtype):
    offsets = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    v = _inputs(len(cuts) - 1, (rows,), 40, 4, dtype)
    y = torch.full_like(v["x"], 99.0)
    _check_forward(v, "silu", (rows,), offsets, y=y)
    assert bool((y[:cuts[0]] == 99).all()) and bool((y[cuts[-1]:] == 99).all())
    _check_grad(v, "silu", (rows,), offsets)
    dx = torch.full_like(v["x"], 99.0)
    block.causal_conv_grad(v["x"], v["x"], v["w"], offsets=offsets, want=("dx",), out={"dx": dx})
    assert bool((dx[:cuts[0]] == 99).all()) and bool((dx[cuts[-1]:] == 99).all())


def test_many_short_sequences():
    lengths = torch.randint(0, 4, (5000,), generator=torch.Generator().manual_seed(5))
    cuts = [0, *lengths.cumsum(0).tolist()]
    offsets = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    v = _inputs(len(cuts) - 1, (cuts[-1],), 10, 4, F)
    _check_forward(v, "silu", (cuts[-1],), offsets)
    _check_grad(v, "silu", (cuts[-1],), offsets)


def test_without_bias_and_window():
    v = _inputs(2, (2, 21), 24, 4, torch.float16, window=False)
    v["bias"] = None
    _check_forward(v, "silu", (2, 21))
    _check_grad(v, "silu", (2, 21))


@pytest.mark.parametrize("off", [0, 1, 2, 8])
def test_slices_of_wider_rows(off):
    wide = torch.randn((3, 40, 100), device=DEV).bfloat16()
    v = _inputs(3, (3, 40), 48, 4, torch.bfloat16)
    v["x"] = wide[..., off:off + 48]
    out = torch.full((3, 40, 100), 5.0, device=DEV).bfloat16()
    _check_forward(v, "silu", (3, 40), y=out[..., off:off + 48])
    assert bool((out[..., :off] == 5).all()) and bool((out[..., off + 48:] == 5).all())
    _check_grad(v, "silu", (3, 40))
    # input and output beside one another in the same rows
    both = torch.randn((3, 40, 96), device=DEV).bfloat16()
    v["x"] = both[..., :48]
    want = block.causal_conv(v["x"].clone(), v["w"], v["bias"], act="silu")
    assert torch.equal(block.causal_conv(v["x"], v["w"], v["bias"], act="silu", y=both[..., 48:]), want)
    # and the tokens in front of the batch: [tokens, batch, channels]
    turned = torch.randn((40, 3, 48), device=DEV).bfloat16().transpose(0, 1)
    v["x"] = turned
    _check_forward(v, "none", (3, 40))


@pytest.mark.parametrize("tokens", [1, 2, 3, 50])
def test_window_in_place_and_a_prompt_in_two_calls(tokens):
    v = _inputs(2, (2, 60), 17, 4, torch.bfloat16)
    whole = _check_forward(dict(v), "silu", (2, 60), state_out=None)
    state = v["state"].clone()
    a = block.causal_conv(v["x"][:, :tokens], v["w"], v["bias"], act="silu", state=state, state_out=state)
    b = block.causal_conv(v["x"][:, tokens:], v["w"], v["bias"], act="silu", state=state, state_out=state)
    assert torch.equal(torch.cat([a, b], 1), whole)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch, d, taps", [(1, 1, 2), (3, 33, 3), (7, 256, 4), (200, 64, 4)])
def test_step_gives_what_the_prompt_gives(batch, d, taps, dtype):
    v = _inputs(batch, (batch, 6), d, taps, dtype)
    whole = block.causal_conv(v["x"], v["w"], v["bias"], act="silu", state=v["state"])
    state = v["state"].clone()
    for t in range(6):
        y = block.causal_conv_step(v["x"][:, t], v["w"], state, v["bias"], act="silu")
        assert torch.equal(y, whole[:, t])
    assert torch.equal(state, torch.cat([v["state"], v["x"]], 1)[:, -(taps - 1):])


def test_no_sequences_and_no_tokens():
    v = _inputs(0, (0, 5), 8, 4, torch.bfloat16)
    assert block.causal_conv(v["x"], v["w"], v["bias"], state=v["state"]).shape == (0, 5, 8)
    g = block.causal_conv_grad(v["x"], v["x"], v["w"], v["bias"])
    assert not g["dw"].any() and not g["dbias"].any()
    v = _inputs(2, (2, 0), 8, 4, torch.bfloat16)
    last = torch.empty_like(v["state"])
    block.causal_conv(v["x"], v["w"], state=v["state"], state_out=last)
    assert torch.equal(last, v["state"])
    g = block.causal_conv_grad(v["x"], v["x"], v["w"], v["bias"], state=v["state"], dstate_out=v["state"])
    assert torch.equal(g["dstate"], v["state"]) and not g["dw"].any()


def test_nan_stays_in_its_channel_and_window():
    v = _inputs(1, (1, 20), 8, 4, torch.float32)
    v["x"][0, 5, 3] = float("nan")
    y = block.causal_conv(v["x"], v["w"], v["bias"], act="silu", state=v["state"])
    bad = torch.isnan(y[0])
    assert bad[5:9, 3].all() and int(bad.sum()) == 4


def test_the_same_bits_again_and_on_another_stream():
    v = _inputs(3, (3, 200), 72, 4, torch.bfloat16)
    dy = torch.randn((3, 200, 72), device=DEV).bfloat16()
    first = block.causal_conv_grad(dy, v["x"], v["w"], v["bias"], act="silu", state=v["state"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = block.causal_conv_grad(dy, v["x"], v["w"], v["bias"], act="silu", state=v["state"], stream=side)
    side.synchronize()
    for k in first:
        assert torch.equal(first[k], again[k]), k
