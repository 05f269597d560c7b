"""Calls at the edges of what include/ttc_block.h allows: no rows with every output there, rows that lie on 16 bytes and no more."""
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import block_util as bu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = torch.float32


@pytest.mark.parametrize("act", [0, 2])
def test_gradients_of_no_rows_with_every_output_there(act):
    """What a caller with buffers of its own hands over for an empty batch: dx stays as it was, the sums are zero."""
    k, m = 32, 48
    w = torch.ones((m, k), device=DEV, dtype=torch.bfloat16)
    dx, dw, dbias = torch.full((4, k), 5.0, device=DEV).bfloat16(), torch.full((m, k), 5.0, device=DEV).bfloat16(), torch.full((m,), 5.0, device=DEV)
    pre = torch.ones((4, m), device=DEV, dtype=torch.bfloat16)
    lib = block._load()
    record = block._LINEAR_ARGS.pack(0, k, m, block.TTC_BF16, block.TTC_BF16, act, 0, w.data_ptr(), w.data_ptr(), 0, 0, 0, pre.data_ptr(), k, k, 0, 0, m)
    grads = block._LINEAR_GRADS.pack(pre.data_ptr(), dx.data_ptr(), dw.data_ptr(), dbias.data_ptr(), m, k, k)
    need = lib.ttc_linear_grad_workspace(0, record, grads)
    assert need >= 0
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    assert lib.ttc_linear_grad(0, record, grads, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert bool((dx == 5).all()) and not dw.any() and not dbias.any()


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("at, width", [(4, 72), (4, 76), (0, 68), (12, 80), (1, 65)])
def test_gradients_of_float32_slices(act, at, width):
    """dy in float32 that begins 16 bytes into a wider row, or whose rows lie 16 bytes off 32: the same bits as from dense rows.  Rows
    off 16 bytes are read column by column and added up in another order: rows + 8 roundings on either side, slopes below 1.13."""
    g = torch.Generator(device=DEV).manual_seed(12)
    rows, k, m = 77, 40, 64
    r = lambda *s, t=torch.bfloat16: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    x, w, pre = r(rows, k), r(m, k), None if act == "none" else r(rows, m)
    wide = r(rows, width, t=F)
    dy = wide[:, at:at + m]
    for keys in (("dx", "dw", "dbias"), ("dbias",)):
        want = block.linear_grad(dy.contiguous(), x, w, act=act, pre=pre, want=keys)
        got = block.linear_grad(dy, x, w, act=act, pre=pre, want=keys)
        for key in keys:
            if key == "dbias" and (at % 4 or width % 4):
                assert bool(((got[key] - want[key]).abs() <= 2 * (rows + 8) * bu.U * 1.13 * dy.abs().sum(0)).all())
            else:
                assert torch.equal(got[key], want[key]), key
    assert block.device_error(0) == 0


def test_wrong_offsets_that_ask_for_more_pieces_than_32_bits_count(monkeypatch):
    """1024 offsets that jump back and forth over 2^28 rows: 512 sequences of all the rows, 2^31 pieces of 64.  The first one has
    its pieces, the others what is left of the room; scratch and outputs stay within their bounds."""
    T, batch = (1 << 28) + 64, 1023
    bf = torch.bfloat16
    one, none = torch.ones((T, 1), device=DEV, dtype=bf), torch.zeros((T, 1), device=DEV, dtype=bf)
    offsets = torch.zeros(batch + 1, device=DEV, dtype=torch.int32)
    offsets[1::2] = T
    kept = []

    def guarded(need, x, stream):
        block._check(min(need, 0))
        kept.append((torch.full((need + 512,), 0x5a, dtype=torch.uint8, device=DEV), need))
        return kept[-1][0], kept[-1][0].data_ptr() + 256

    monkeypatch.setattr(block, "_workspace", guarded)
    A, last = torch.full((1, 1), -0.5, device=DEV), torch.ones((batch, 1, 1), device=DEV)
    got = block.selective_scan_grad(none, one, none, A, one, one, offsets=offsets, dstate_out=last, want=("dA", "dstate", "ddelta_bias"))
    torch.cuda.synchronize()
    for ws, need in kept:
        assert bool((ws[:256] == 0x5a).all()) and bool((ws[256 + need:] == 0x5a).all())
    assert float(got["dstate"][0]) == 1.0                            # steps of zero: nothing decays, and dy is zero
    assert torch.isfinite(got["dA"]).all() and not got["dA"].any()   # no step, no share


@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("n", [16, 6])
def test_a_decay_of_minus_infinity_in_single_tokens(n, softplus):
    """What the prompt gives: a step of nothing (of zero, or a softplus below the numbers there are) keeps the state, any other
    leaves the token's share.  Either side is off by at most 24 operations a token, of the magnitudes that were ever added."""
    g = torch.Generator(device=DEV).manual_seed(14)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    batch, d = 3, 10
    x, B, C, D, delta = r(batch, 4, d), r(batch, 4, n), r(batch, 4, n), r(d), r(batch, 4, d).abs()
    delta[:, 1::2] = -200.0 if softplus else 0.0
    A = -torch.rand((d, n), generator=g, device=DEV)
    A[4], A[7, 1] = float("-inf"), float("-inf")
    state = r(batch, d, n)
    last, mag = torch.empty_like(state), state.abs()
    y = block.selective_scan(x, delta, A, B, C, D=D, softplus=softplus, state=state, state_out=last)
    steps = torch.nn.functional.softplus(delta) if softplus else delta
    assert torch.isfinite(y).all() and torch.isfinite(last).all()
    for t in range(4):
        before = state.clone()
        got = block.selective_scan_step(x[:, t], delta[:, t], A, B[:, t], C[:, t], state, D=D, softplus=softplus)
        if t % 2:
            assert torch.equal(state, before)
        mag = mag + (steps[:, t] * x[:, t]).abs()[..., None] * B[:, t, None].abs()
        room = 2 * (n + 24 * (t + 1)) * bu.U * ((mag * C[:, t, None].abs()).sum(-1) + (D * x[:, t]).abs())
        assert bool(((got - y[:, t]).abs() <= room).all()), t
    assert bool(((state - last).abs() <= 2 * 24 * 4 * bu.U * mag).all())
    share = (torch.nn.functional.softplus(delta[:, 2, 4].double()) if softplus else delta[:, 2, 4].double()) * x[:, 2, 4].double()
    want = share[:, None] * B[:, 2].double()
    assert bool(((state[:, 4].double() - want).abs() <= 24 * bu.U * want.abs()).all())


@pytest.mark.parametrize("dtype", [F, torch.bfloat16])
@pytest.mark.parametrize("act", ["relu", "silu", "gelu", "softplus"])
def test_each_gradient_of_an_activation_alone_has_the_same_bits(act, dtype):
    g = torch.Generator(device=DEV).manual_seed(15)
    r = lambda *s, t=torch.bfloat16: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    for rows, k, m in ((77, 40, 64), (301, 33, 45)):
        x, w, pre, dy = r(rows, k), r(m, k), r(rows, m), r(rows, m, t=dtype)
        whole = block.linear_grad(dy, x, w, act=act, pre=pre)
        for key in whole:
            assert torch.equal(block.linear_grad(dy, x, w, act=act, pre=pre, want=(key,))[key], whole[key]), key


def test_outputs_in_other_tokens_of_the_inputs_storage():
    g = torch.Generator(device=DEV).manual_seed(16)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    for batch in (1, 3):
        room, d, n = r(batch, 130, 24), 24, 8
        x, y = room[:, :65], room[:, 65:]
        taps, A, B = r(d, 4), -r(d, n).abs(), r(batch, 65, n)
        want = block.causal_conv(x.clone(), taps, act="silu")
        assert torch.equal(block.causal_conv(x, taps, act="silu", y=y), want)
        want = block.selective_scan(x.clone(), x.clone(), A, B, B, softplus=True)
        assert torch.equal(block.selective_scan(x, x, A, B, B, softplus=True, y=y), want)
        dy = r(batch, 65, d)
        want = block.causal_conv_grad(dy, x.clone(), taps, want=("dx",))["dx"]
        assert torch.equal(block.causal_conv_grad(dy, x, taps, want=("dx",), out={"dx": y})["dx"], want)
        with pytest.raises(Exception, match="overlap"):
            block.causal_conv(x, taps, y=room[:, 64:129])


@pytest.mark.parametrize("rows", [5, 70])
def test_one_row_for_all_tokens(rows):
    """Operands of projections that are the same row again and again (expand), or rows that lie over one another, as the others:
    the same bits as from copies, on the current stream and on a named one."""
    g = torch.Generator(device=DEV).manual_seed(17)
    r = lambda *s, t=torch.bfloat16: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    k, m = 40, 24
    x, w, res, dy, pre = r(rows, k), r(m, k), r(rows, m), r(rows, m), r(rows, m)
    line = r(16 * max(rows, m) + k)
    again = dict(x=x[:1].expand(rows, k), w=w[:1].expand(m, k), residual=res[:1].expand(rows, m), dy=dy[:1].expand(rows, m), pre=pre[:1].expand(rows, m))
    over = dict(x=line.as_strided((rows, k), (8, 1)), w=line.as_strided((m, k), (8, 1)), residual=line.as_strided((rows, m), (1, 1)),
                dy=line.as_strided((rows, m), (16, 1)), pre=line.as_strided((rows, m), (8, 1)))
    batched = dict(x=x[None, :1].expand(rows, 2, k)[:, 0], residual=res[None].expand(2, rows, m)[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for some in (again, over, batched):
        for name, t in some.items():
            a = {**dict(x=x, w=w, residual=res, dy=dy, pre=pre), name: t}
            b = {**a, name: t.contiguous()}
            for stream in (None, side):
                forward = lambda v: block.linear(v["x"], v["w"], residual=v["residual"], act="silu", stream=stream)  # noqa: E731
                back = lambda v: block.linear_grad(v["dy"], v["x"], v["w"], act="silu", pre=v["pre"], stream=stream)  # noqa: E731
                torch.cuda.synchronize()
                assert torch.equal(forward(a), forward(b)), name
                one, two = back(a), back(b)
                side.synchronize()
                assert all(torch.equal(one[q], two[q]) for q in one), name
    with pytest.raises(Exception):                                   # but no output
        block.linear(x, w, y=res[:1].expand(rows, m))


def test_rows_past_32_bits():
    """Rows whose elements lie more than 2^31 behind the first: the last tokens are what a call on them alone gives, from the window and
    state in front of them.  (A state that begins 4000 tokens earlier has forgotten, at decays below exp(-0.2 D), what was before.)"""
    g = torch.Generator(device=DEV).manual_seed(18)
    r = lambda *s, t=torch.bfloat16: torch.randn(s, generator=g, device=DEV, dtype=t)  # noqa: E731
    T, d, n = 530000, 4096, 4
    assert (T - 1000) * d > 2 ** 31
    x, taps, A, B = r(1, T, d), r(d, 4, t=F), -torch.rand((d, n), generator=g, device=DEV) - 0.2, r(1, T, n)
    y = block.causal_conv(x, taps, act="silu")
    tail, before = (lambda t: t[:, T - 1000:].contiguous()), (lambda t: t[:, T - 5000:T - 1000].contiguous())  # noqa: E731
    window = x[:, T - 1003:T - 1000].contiguous()
    assert torch.equal(tail(y), block.causal_conv(tail(x), taps, act="silu", state=window))
    dx = block.causal_conv_grad(y, x, taps, act="silu", want=("dx",))["dx"]
    assert torch.equal(tail(dx), block.causal_conv_grad(tail(y), tail(x), taps, act="silu", state=window, want=("dx",))["dx"])
    state, last, end = (torch.empty((1, d, n), device=DEV) for _ in range(3))
    block.selective_scan(before(x), before(y), A, before(B), before(B), softplus=True, state_out=state)
    want = block.selective_scan(tail(x), tail(y), A, tail(B), tail(B), softplus=True, state=state, state_out=last)
    out = block.selective_scan(x, y, A, B, B, softplus=True, state_out=end, y=dx)
    close = lambda a, b, limit: float((a.double() - b.double()).norm() / b.double().norm()) <= limit  # noqa: E731
    assert close(tail(out), want, 1e-4) and close(end, last, 1e-6)   # (a rounding to bfloat16 that falls the other way now and then)
    del out, dx
    got = block.selective_scan_grad(y, x, y, A, B, B, softplus=True, want=("ddelta", "dB"))
    want = block.selective_scan_grad(tail(y), tail(x), tail(y), A, tail(B), tail(B), softplus=True, state=state, want=("ddelta", "dB"))
    for key in want:
        assert close(tail(got[key]), want[key], 1e-4), key


def test_projections_past_32_bits():
    g = torch.Generator(device=DEV).manual_seed(19)
    r = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    rows, k, m = 70001, 64, 32776
    x, w, res = r(rows, k), r(m, k), r(rows, m)
    end = slice(rows - 300, rows)
    assert end.start * m > 2 ** 31
    assert torch.equal(block.linear(x, w, residual=res, act="silu")[end], block.linear(x[end], w, residual=res[end], act="silu"))
    dx, want = block.linear_grad(res, x, w, want=("dx",))["dx"][end].double(), res[end].double() @ w.double()
    # half a step of bfloat16, and 2 u of the magnitudes for each 16 of the products
    room = 2.0 ** -8 * want.abs() + 2 * bu.U * (m / 16 + 8) * (res[end].double().abs() @ w.double().abs())
    assert bool(((dx - want).abs() <= room).all()) and block.device_error(0) == 0


def test_calls_from_several_threads():
    """Each thread on a stream of its own, with its own states: single tokens, projections and gradients at once."""
    import threading
    bf = torch.bfloat16

    def work(seed, out):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s, t=bf: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
        x, w, taps, A, B = r(6, 64), r(64, 64) * 0.125, r(64, 4, t=F) * 0.5, -r(64, 16, t=F).abs(), r(6, 16) * 0.25
        window, state = torch.zeros((6, 3, 64), device=DEV, dtype=bf), torch.zeros((6, 64, 16), device=DEV)
        got = []
        for _ in range(40):
            c = block.causal_conv_step(block.linear(x, w), taps, window, act="silu")
            x = block.linear(block.selective_scan_step(c, c, A, B, B, state, softplus=True), w, residual=x) * 0.1
            got += [x, block.linear_grad(x, c, w)["dw"], block.selective_scan_grad(x[None], c[None], c[None], A, B[None], B[None], softplus=True)["dA"]]
        torch.cuda.current_stream().synchronize()
        out[seed] = [*got, window, state]

    def on_a_stream(seed, out):
        with torch.cuda.stream(torch.cuda.Stream()):
            work(seed, out)

    alone, together = {}, {}
    for seed in range(4):
        work(seed, alone)
    threads = [threading.Thread(target=on_a_stream, args=(seed, together)) for seed in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert sorted(together) == sorted(alone)
    for seed in alone:
        assert all(torch.isfinite(a).all() and torch.equal(a, b) for a, b in zip(alone[seed], together[seed])), seed
