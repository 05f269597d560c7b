"""The operators of the block around the Test-Time Control layer, as cases that can be timed and compared: projections of
token rows (with bias, activation and residual), the short causal convolution, and the selective state space scan, each
forward, backward and, where a model decodes, for single tokens.

``run`` computes a case in its plain form, in elementary torch operations in 32 bits, or, where ``own`` is true, by the
calls of ``paper_2603_09221_b200.block`` that a program makes.  Notation: ``T`` token rows (of one batch of equal
sequences, or packed one behind the other with ``offsets``), ``d`` channels, ``n`` states per channel, ``g`` groups of
channels that share ``B`` and ``C``, ``w`` taps of the convolution.

  linear        y = act(x W' + b) + r                                       x [T, k], W [m, k]
  linear_grad   dZ = dy act'(z);  dx = dZ W,  dW = dZ' x,  db = sum_t dZ
  conv          y_t = silu(b + sum_j w_j x_{t-(w-1)+j}), the window in front of a sequence given, the last one returned
  scan          D_t = softplus(delta_t + bias);  h_t = exp(D_t A) h_{t-1} + D_t x_t B_t;
                y_t = (C_t . h_t + D x_t) silu(z_t), the state in front of a sequence given, the last one returned
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GRAD_OPS = ("linear_grad", "conv_grad", "scan_grad")


def _linear(op, rows, k, m, dtype, act, residual=False, out="same", name=None):
    c = dict(op=op, rows=rows, k=k, m=m, dtype=dtype, act=act)
    if op == "linear":
        c.update(residual=residual, out=out)
    return c if name is None else dict(c, name=name)


def _conv(op, batch, tokens, d, dtype, w=4, packed=False, name=None):
    c = dict(op=op, batch=batch, tokens=tokens, d=d, dtype=dtype, w=w)
    if op != "conv_step":
        c.update(packed=packed)
    return c if name is None else dict(c, name=name)


def _scan(op, batch, tokens, d, n, dtype, g=1, packed=False, name=None):
    c = dict(op=op, batch=batch, tokens=tokens, d=d, n=n, dtype=dtype, g=g)
    if op != "scan_step":
        c.update(packed=packed)
    return c if name is None else dict(c, name=name)


def listed():
    # `tokens` counts the tokens of all sequences together where they are packed, else those of one sequence.
    return [
        # Decoding: one new token of each of 8 sequences through a projection of the block.
        _linear("linear", 8, 2048, 4096, "bf16", "silu", name="linear_decode"),
        # The coefficient vectors that the control layer is handed, for 4 sequences of 1024 tokens: 16 heads of 16 states
        # with 16 basis matrices, 9 vectors each; the layer reads float32, and its gates are softplus outputs.
        _linear("linear", 4096, 1024, 2304, "bf16", "softplus", out="f32", name="linear_coefficients"),
        # The output projection of a prompt of ragged length, added to the residual stream.
        _linear("linear", 8189, 4096, 2048, "f16", "none", residual=True, name="linear_residual"),
        # Training: the gradients of a wide projection over 4 sequences of 2048 tokens.
        _linear("linear_grad", 8192, 2048, 8192, "bf16", "gelu", name="linear_train"),
        # Decoding: the convolution's window moves on by one token, 64 sequences.
        _conv("conv_step", 64, 1, 4096, "bf16", name="conv_decode"),
        # Prompts of 2048 tokens, 4 sequences.
        _conv("conv", 4, 2048, 4096, "bf16", name="conv_prefill"),
        # Training on 11 documents of different lengths packed into 8191 rows, odd number of channels.
        _conv("conv_grad", 11, 8191, 2047, "bf16", packed=True, name="conv_train_packed"),
        # Decoding: 16 sequences, one token each; the state is float32.
        _scan("scan_step", 16, 1, 4096, 16, "bf16", name="scan_decode"),
        # Prompts of 2048 tokens, 4 sequences: enough channels for every SM.
        _scan("scan", 4, 2048, 4096, 16, "bf16", name="scan_prefill"),
        # One long prompt of odd length: few channels, the work is in the tokens.
        _scan("scan", 1, 16381, 1024, 16, "f16", name="scan_long"),
        # Packed documents in float32, more states, two groups.
        _scan("scan", 7, 4093, 1024, 64, "f32", g=2, packed=True, name="scan_packed_n64"),
        # Training: every gradient of 4 sequences of 1024 tokens.
        _scan("scan_grad", 4, 1024, 2048, 16, "bf16", name="scan_train"),
    ]


def _spread(rng, low, high):
    """A whole number between the two, evenly over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(("linear", "linear", "linear_grad", "conv_step", "conv", "conv_grad", "scan_step", "scan", "scan", "scan_grad"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op.startswith("linear"):
        dtype = "f16" if dtype == "f32" else dtype
        rows, k, m = _spread(rng, 1, 8192), _spread(rng, 64, 4096), _spread(rng, 16, 8192)
        if rng.random() < 0.5:                                  # widths of models are multiples of 64; odd ones are served too
            k, m = -(-k // 64) * 64, -(-m // 64) * 64
        act = rng.choice(("none", "relu", "silu", "gelu", "softplus"))
        return _linear(op, rows, k, m, dtype, act, residual=rng.random() < 0.3, out=rng.choice(("same", "same", "f32")))
    d = _spread(rng, 64, 4096)
    d = d if rng.random() < 0.4 else -(-d // 64) * 64
    if op == "conv_step":
        return _conv(op, _spread(rng, 1, 512), 1, d, dtype, w=rng.choice((2, 3, 4)))
    if op.startswith("conv"):
        packed = rng.random() < 0.4
        batch = _spread(rng, 1, 16)
        tokens = _spread(rng, 32, 16384)
        return _conv(op, batch, tokens if packed else max(1, tokens // batch), d, dtype, w=rng.choice((2, 3, 4)), packed=packed)
    n = rng.choice((4, 8, 16, 16, 16, 24, 32, 64))
    g = rng.choice((1, 1, 1, 2, 4))
    d = -(-d // g) * g
    if op == "scan_step":
        return _scan(op, _spread(rng, 1, 512), 1, d, n, dtype, g=g)
    packed = rng.random() < 0.4
    batch = _spread(rng, 1, 16)
    most = (4 * 2048 * 4096 * 16 if op == "scan" else 4 * 1024 * 2048 * 16) // (d * n)     # no more than the largest listed
    tokens = min(most, _spread(rng, 32, 16384))
    return _scan(op, batch, tokens if packed else max(1, tokens // batch), d, n, dtype, g=g, packed=packed)


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _offsets(gen, batch, rows):
    """Offsets of `batch` sequences of different lengths that fill `rows` rows."""
    cuts = torch.randint(0, rows + 1, (batch - 1,), generator=gen, device=DEVICE).sort().values
    edge = torch.zeros(1, dtype=cuts.dtype, device=DEVICE)
    return torch.cat([edge, cuts, edge + rows]).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    t = DTYPES[case["dtype"]]

    def randn(*shape, scale=1.0, dtype=t):
        return (torch.randn(shape, generator=gen, device=DEVICE) * scale).to(dtype)

    s = dict(case=case)
    op = case["op"]
    if op.startswith("linear"):
        rows, k, m = case["rows"], case["k"], case["m"]
        s.update(x=randn(rows, k), w=randn(m, k, scale=k ** -0.5))
        if op == "linear":
            s["out"] = t if case["out"] == "same" else torch.float32
            s.update(bias=randn(m, scale=0.1, dtype=torch.float32))
            s["residual"] = randn(rows, m, dtype=s["out"]) if case["residual"] else None
        else:
            s.update(dy=randn(rows, m), pre=randn(rows, m) if case["act"] != "none" else None)
        return s
    batch, d = case["batch"], case["d"]
    packed = case.get("packed", False)
    rows = case["tokens"] if packed else batch * case["tokens"]
    lead = (rows,) if packed or op.endswith("_step") else (batch, case["tokens"])
    s["offsets"] = _offsets(gen, batch, rows) if packed else None
    s["lead"] = lead
    if op.startswith("conv"):
        w = case["w"]
        s.update(x=randn(*lead, d), w=randn(d, w, scale=w ** -0.5, dtype=torch.float32), bias=randn(d, scale=0.1, dtype=torch.float32),
                 state=randn(batch, w - 1, d))
        if op == "conv_grad":
            s.update(dy=randn(*lead, d), dstate_out=randn(batch, w - 1, d))
        return s
    n, g = case["n"], case["g"]
    # decay rates 1 .. n per channel, step sizes between 1e-3 and 1e-1 (softplus of what a projection gives plus a bias)
    step = torch.exp(torch.rand(d, generator=gen, device=DEVICE) * math.log(100.0) + math.log(1e-3))
    s.update(A=-(torch.arange(1, n + 1, device=DEVICE) * (1 + 0.1 * torch.rand((d, n), generator=gen, device=DEVICE))).float(),
             delta_bias=step + torch.log(-torch.expm1(-step)), delta=randn(*lead, d, scale=0.5), x=randn(*lead, d), z=randn(*lead, d),
             B=randn(*lead, g, n), C=randn(*lead, g, n), D=randn(d, dtype=torch.float32), state=randn(batch, d, n, scale=0.3, dtype=torch.float32))
    if op == "scan_grad":
        s.update(dy=randn(*lead, d), dstate_out=randn(batch, d, n, dtype=torch.float32))
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "softplus":
        return z.clamp(min=0) + torch.log1p(torch.exp(-z.abs()))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    p = 1 / (1 + torch.exp(-z))
    if act == "silu":
        return p * (1 + z * (1 - p))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return p                                                    # softplus


def _plain_linear(s):
    z = s["x"].float() @ s["w"].float().t() + s["bias"]
    y = _act(z, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(s["out"])}


def _plain_linear_grad(s):
    dz = s["dy"].float()
    if s["pre"] is not None:
        dz = dz * _act_slope(s["pre"].float(), s["case"]["act"])
    return {"dx": (dz @ s["w"].float()).to(s["x"].dtype), "dw": (dz.t() @ s["x"].float()).to(s["w"].dtype), "dbias": dz.sum(0)}


def _bounds(s):
    """First and one-past-last row of every sequence among the flattened rows, and the longest sequence's length at most."""
    if s["offsets"] is not None:
        o = s["offsets"].long()
        return o[:-1], o[1:], s["lead"][0]
    batch, tokens = s["lead"]
    first = torch.arange(batch, device=DEVICE) * tokens
    return first, first + tokens, tokens


def _place(first, end, rows):
    """Sequence of every row and its index in it."""
    row = torch.arange(rows, device=DEVICE)
    seq = torch.searchsorted(end, row, right=True)
    return seq, row - first[seq]


def _taps(s):
    """The conv's inputs x_{t-(w-1)+j}, j = 0..w-1, as [w, rows, d] in 32 bits: from the rows, or from the window in front."""
    x = s["x"].float().flatten(0, -2)
    first, end, _ = _bounds(s)
    seq, at = _place(first, end, x.shape[0])
    back = torch.arange(s["case"]["w"] - 1, -1, -1, device=DEVICE)[:, None]                   # rows to go back
    row = (torch.arange(x.shape[0], device=DEVICE)[None] - back).clamp(min=0)
    window = s["state"].float()[seq[None], (at[None] - back).remainder(max(1, s["case"]["w"] - 1))]
    inside = (at[None] >= back)[..., None]
    # tap at - back < 0 lies in the window at place (w - 1) + at - back, which the remainder gives
    return torch.where(inside, x[row], window)


def _window_rows(s):
    """Where the last w - 1 inputs of every sequence lie: row among the rows (or -1) and place in the window in front."""
    w = s["case"]["w"]
    first, end, _ = _bounds(s)
    back = torch.arange(w - 1, 0, -1, device=DEVICE)[None]
    at = (end - first)[:, None] - back                                                        # index in the sequence
    return torch.where(at >= 0, first[:, None] + at, -1), (at + w - 1).clamp(max=w - 2)


def _plain_conv(s):
    taps = _taps(s)
    z = s["bias"] + (taps * s["w"].t()[:, None, :]).sum(0)
    row, place = _window_rows(s)
    x = s["x"].flatten(0, -2)
    kept = torch.gather(s["state"], 1, place[..., None].expand(-1, -1, x.shape[1]))
    return {"y": _act(z, "silu").to(s["x"].dtype).reshape(s["x"].shape), "state_out": torch.where((row >= 0)[..., None], x[row.clamp(min=0)], kept)}


def _plain_conv_step(s):
    taps = torch.cat([s["state"], s["x"][:, None]], 1)
    z = s["bias"] + (taps.float() * s["w"].t()[None]).sum(1)
    s["state"].copy_(taps[:, 1:])
    return {"y": _act(z, "silu").to(s["x"].dtype), "state": s["state"]}


def _plain_conv_grad(s):
    w = s["case"]["w"]
    taps = _taps(s)
    d = taps.shape[2]
    z = s["bias"] + (taps * s["w"].t()[:, None, :]).sum(0)
    dz = s["dy"].float().flatten(0, -2) * _act_slope(z, "silu")
    dw, dbias = (taps * dz[None]).sum(1).t(), dz.sum(0)
    rows = z.shape[0]
    first, end, _ = _bounds(s)
    seq, at = _place(first, end, rows)
    # every tap hands its share to a row or, in front of the sequence, to the window
    back = torch.arange(w - 1, -1, -1, device=DEVICE)[:, None]
    share = dz[None] * s["w"].t()[:, None, :]
    inside = at[None] >= back
    row = torch.where(inside, torch.arange(rows, device=DEVICE)[None] - back, rows)            # `rows`: a row for the rest
    dx = torch.zeros(rows + 1, d, device=DEVICE).index_add_(0, row.flatten(), share.flatten(0, 1))
    slot = torch.where(inside, s["state"].shape[0] * (w - 1), seq[None] * (w - 1) + at[None] - back + w - 1)
    dstate = torch.zeros(s["state"].shape[0] * (w - 1) + 1, d, device=DEVICE).index_add_(0, slot.flatten(), share.flatten(0, 1))
    row, place = _window_rows(s)                                                              # and the last window's gradient
    last = s["dstate_out"].float()
    dx.index_add_(0, torch.where(row >= 0, row, rows).flatten(), last.flatten(0, 1))
    slot = torch.where(row >= 0, s["state"].shape[0] * (w - 1), torch.arange(row.shape[0], device=DEVICE)[:, None] * (w - 1) + place)
    dstate.index_add_(0, slot.flatten(), last.flatten(0, 1))
    return {"dx": dx[:rows].to(s["x"].dtype).reshape(s["x"].shape), "dw": dw.contiguous(), "dbias": dbias,
            "dstate": dstate[:-1].reshape(s["state"].shape).to(s["x"].dtype)}


def _doubling(a, b, longest):
    """h_t = a_t h_{t-1} + b_t along the first axis, from h = 0, in ceil(log2(longest)) rounds; a and b are overwritten."""
    reach = 1
    while reach < longest:
        b[reach:] += a[reach:] * b[:-reach]
        a[reach:] = a[reach:] * a[:-reach]
        reach *= 2
    return b


def _spread_groups(v, d):
    """[rows, g, n] -> [rows, d, n]: the group of every channel."""
    return v.float().repeat_interleave(d // v.shape[1], 1)


def _plain_scan_parts(s):
    f = lambda k: s[k].float().flatten(0, len(s["lead"]) - 1)  # noqa: E731
    x, z = f("x"), f("z")
    raw = f("delta") + s["delta_bias"]
    step = _act(raw, "softplus")
    B, C = _spread_groups(f("B"), x.shape[1]), _spread_groups(f("C"), x.shape[1])
    a = torch.exp(step[..., None] * s["A"])
    b = (step * x)[..., None] * B
    first, end, longest = _bounds(s)
    some = end > first                                          # packed sequences may be empty
    return x, z, raw, step, B, C, a, b, first, end, some, longest


def _plain_scan(s):
    x, z, raw, step, B, C, a, b, first, end, some, longest = _plain_scan_parts(s)
    b[first[some]] += a[first[some]] * s["state"][some]
    a[first[some]] = 0
    h = _doubling(a, b, longest)
    y = ((h * C).sum(-1) + s["D"] * x) * _act(z, "silu")
    last = torch.where(some[:, None, None], h[(end - 1).clamp(min=0)], s["state"])
    return {"y": y.to(s["x"].dtype).reshape(s["x"].shape), "state_out": last}


def _plain_scan_step(s):
    x, z = s["x"].float(), s["z"].float()
    step = _act(s["delta"].float() + s["delta_bias"], "softplus")
    B, C = _spread_groups(s["B"], x.shape[1]), _spread_groups(s["C"], x.shape[1])
    s["state"].mul_(torch.exp(step[..., None] * s["A"])).add_((step * x)[..., None] * B)
    y = ((s["state"] * C).sum(-1) + s["D"] * x) * _act(z, "silu")
    return {"y": y.to(s["x"].dtype), "state": s["state"]}


def _plain_scan_grad(s):
    x, z, raw, step, B, C, a, b, first, end, some, longest = _plain_scan_parts(s)
    rows, d, n = a.shape
    g = s["B"].shape[-2]
    f, l = first[some], end[some] - 1
    b[f] += a[f] * s["state"][some]
    a0 = a.clone()
    a0[f] = 0
    h = _doubling(a0, b, longest)
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[f] = s["state"][some]
    dy = s["dy"].float().flatten(0, len(s["lead"]) - 1)
    gated = dy * _act(z, "silu")
    dz = dy * ((h * C).sum(-1) + s["D"] * x) * _act_slope(z, "silu")
    # co-states: q_t = C_t gated_t + a_{t+1} q_{t+1}, from the gradient of the last state
    q = gated[..., None] * C
    q[l] += s["dstate_out"][some]
    later = torch.cat([a[1:], torch.zeros_like(a[:1])])
    later[l] = 0
    q = _doubling(later.flip(0), q.flip(0), longest).flip(0)
    dstate = s["dstate_out"].clone()
    dstate[some] = a[f] * q[f]
    grouped = lambda v: v.reshape(rows, g, d // g, n).sum(2).to(s["x"].dtype).reshape(s["B"].shape)  # noqa: E731
    dC = grouped(h * gated[..., None])
    dB = grouped(q * (step * x)[..., None])
    qB = (q * B).sum(-1)
    qah = q * a * before
    draw_ = (x * qB + (qah * s["A"]).sum(-1)) * (1 / (1 + torch.exp(-raw)))
    shape = lambda v: v.to(s["x"].dtype).reshape(s["x"].shape)  # noqa: E731
    return {"dx": shape(step * qB + s["D"] * gated), "ddelta": shape(draw_), "dz": shape(dz), "dB": dB, "dC": dC,
            "dA": (qah * step[..., None]).sum(0), "dD": (gated * x).sum(0), "ddelta_bias": draw_.sum(0), "dstate": dstate}


PLAIN = {"linear": _plain_linear, "linear_grad": _plain_linear_grad, "conv": _plain_conv, "conv_step": _plain_conv_step,
         "conv_grad": _plain_conv_grad, "scan": _plain_scan, "scan_step": _plain_scan_step, "scan_grad": _plain_scan_grad}


# ---- the framework's calls --------------------------------------------------------------------------------------------

def _own(s):
    from paper_2603_09221_b200 import block
    op, act = s["case"]["op"], s["case"].get("act")
    if op == "linear":
        return {"y": block.linear(s["x"], s["w"], s["bias"], act=act, residual=s["residual"], out_dtype=s["out"])}
    if op == "linear_grad":
        return block.linear_grad(s["dy"], s["x"], s["w"], act=act, pre=s["pre"])
    if op == "conv":
        state_out = torch.empty_like(s["state"])
        return {"y": block.causal_conv(s["x"], s["w"], s["bias"], act="silu", state=s["state"], offsets=s["offsets"], state_out=state_out),
                "state_out": state_out}
    if op == "conv_step":
        return {"y": block.causal_conv_step(s["x"], s["w"], s["state"], s["bias"], act="silu"), "state": s["state"]}
    if op == "conv_grad":
        return block.causal_conv_grad(s["dy"], s["x"], s["w"], s["bias"], act="silu", state=s["state"], offsets=s["offsets"],
                                      dstate_out=s["dstate_out"])
    args = (s["x"], s["delta"], s["A"], s["B"], s["C"])
    more = dict(D=s["D"], z=s["z"], delta_bias=s["delta_bias"], softplus=True, state=s["state"])
    if op == "scan":
        state_out = torch.empty_like(s["state"])
        return {"y": block.selective_scan(*args, **more, offsets=s["offsets"], state_out=state_out), "state_out": state_out}
    if op == "scan_step":
        return {"y": block.selective_scan_step(*args, **more), "state": s["state"]}
    return block.selective_scan_grad(s["dy"], *args, **more, offsets=s["offsets"], dstate_out=s["dstate_out"])


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    op, size = case["op"], 4 if case["dtype"] == "f32" else 2
    if op.startswith("linear"):
        rows, k, m = case["rows"], case["k"], case["m"]
        if op == "linear":
            out = size if case["out"] == "same" else 4
            return {"bytes": (rows * k + m * k) * size + rows * m * out * (2 if case["residual"] else 1) + 4 * m, "flops": 2 * rows * k * m}
        slope = case["act"] != "none"
        return {"bytes": size * (2 * rows * k + 2 * m * k + rows * m * (2 if slope else 1)) + 4 * m, "flops": 4 * rows * k * m}
    batch, d = case["batch"], case["d"]
    rows = case["tokens"] if case.get("packed") else batch * case["tokens"]
    if op.startswith("conv"):
        w = case["w"]
        window = batch * (w - 1) * d * size
        if op == "conv_grad":
            return {"bytes": 3 * rows * d * size + 3 * window + 8 * d * (w + 1), "flops": rows * d * (6 * w + 10)}
        return {"bytes": 2 * rows * d * size + 2 * window + 4 * d * (w + 1), "flops": rows * d * (2 * w + 4)}
    n, g = case["n"], case["g"]
    states, shared = batch * d * n * 4, rows * g * n * size
    if op == "scan_grad":
        return {"bytes": 7 * rows * d * size + 4 * shared + 3 * states + 8 * d * (n + 2), "flops": rows * d * (18 * n + 20)}
    return {"bytes": 4 * rows * d * size + 2 * shared + 2 * states + 4 * d * (n + 2), "flops": rows * d * (7 * n + 10)}


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------

def _sequences(s):
    """Slices of the flattened rows, one of each sequence."""
    if s["offsets"] is not None:
        o = s["offsets"].tolist()
        return [slice(a, b) for a, b in zip(o[:-1], o[1:])]
    batch, tokens = s["lead"]
    return [slice(i * tokens, (i + 1) * tokens) for i in range(batch)]


def _exact_conv(s, grad):
    size = s["case"]["w"]
    x = s["x"].double().flatten(0, -2).requires_grad_()
    state, w, bias = (s[k].double().requires_grad_() for k in ("state", "w", "bias"))
    ys, last = [], []
    for i, rows in enumerate(_sequences(s)):
        line = torch.cat([state[i], x[rows]])                                                  # the window, then the tokens
        tokens = rows.stop - rows.start
        z = bias + sum(line[j:j + tokens] * w[:, j] for j in range(size))
        ys.append(z * torch.sigmoid(z))
        last.append(line[tokens:])
    y, last = torch.cat(ys), torch.stack(last)
    if not grad:
        return {"y": y.detach(), "state_out": last.detach()}
    loss = (y * s["dy"].double().flatten(0, -2)).sum() + (last * s["dstate_out"].double()).sum()
    dx, dw, dbias, dstate = torch.autograd.grad(loss, (x, w, bias, state))
    return {"dx": dx, "dw": dw, "dbias": dbias, "dstate": dstate}


def _exact_scan(s, grad):
    """Row by row, as the recurrence is written; equal sequences side by side."""
    even = s["offsets"] is None
    batch, tokens = s["lead"] if even else (None, None)
    view = (lambda v: v.double().reshape(batch, tokens, *v.shape[2:])) if even else (lambda v: v.double()[None])
    x, delta, z, B, C = (view(s[k]) for k in ("x", "delta", "z", "B", "C"))
    d, n = s["A"].shape
    A, D = s["A"].double(), s["D"].double()
    raw = delta + s["delta_bias"].double()
    step = torch.logaddexp(raw, torch.zeros_like(raw))
    share = d // B.shape[2]
    gate = z * torch.sigmoid(z)
    wide = lambda v: v[:, :, None].expand(-1, -1, share, -1).reshape(v.shape[0], d, n)  # noqa: E731  (one row's groups)
    spans = [(0, tokens, slice(0, batch))] if even else [(r.start, r.stop, slice(i, i + 1)) for i, r in enumerate(_sequences(s))]
    y = torch.empty_like(x)
    last = s["state"].double().clone()
    hs = torch.empty((x.shape[0], x.shape[1], d, n), dtype=torch.float64, device=x.device) if grad else None
    for lo, hi, who in spans:
        h = s["state"][who].double()
        for t in range(lo, hi):
            h = torch.exp(step[:, t, :, None] * A) * h + (step[:, t] * x[:, t])[..., None] * wide(B[:, t])
            y[:, t] = (h * wide(C[:, t])).sum(-1)
            if grad:
                hs[:, t] = h
        last[who] = h
    out = y + D * x
    flat = lambda v: v.flatten(0, 1)  # noqa: E731
    if not grad:
        return {"y": flat(out * gate), "state_out": last}
    dy = view(s["dy"])
    gated = dy * gate
    p = torch.sigmoid(z)
    dz = dy * out * (p + z * p * (1 - p))
    dx, dstep, dB, dC = D * gated, torch.empty_like(x), torch.empty_like(B), torch.empty_like(C)
    dA, dstate = torch.zeros_like(A), s["dstate_out"].double().clone()
    narrow = lambda v: v.reshape(v.shape[0], -1, share, n).sum(2)  # noqa: E731
    for lo, hi, who in spans:
        q = s["dstate_out"][who].double()
        for t in range(hi - 1, lo - 1, -1):
            q = q + gated[:, t, :, None] * wide(C[:, t])
            before = hs[:, t - 1] if t > lo else s["state"][who].double()
            a = torch.exp(step[:, t, :, None] * A)
            dC[:, t] = narrow(gated[:, t, :, None] * hs[:, t])
            dB[:, t] = narrow(q * (step[:, t] * x[:, t])[..., None])
            qB = (q * wide(B[:, t])).sum(-1)
            through = q * a * before
            dx[:, t] += step[:, t] * qB
            dstep[:, t] = x[:, t] * qB + (through * A).sum(-1)
            dA += (through * step[:, t, :, None]).sum(0)
            q = a * q
        dstate[who] = q
    ddelta = dstep * torch.sigmoid(raw)
    return {"dx": dx, "ddelta": ddelta, "dz": dz, "dB": dB, "dC": dC, "dA": dA, "dD": flat(gated * x).sum(0),
            "ddelta_bias": flat(ddelta).sum(0), "dstate": dstate}


def _exact_act(z, act):
    return {"none": lambda: z, "relu": lambda: torch.relu(z), "silu": lambda: z * torch.sigmoid(z),
            "gelu": lambda: z * torch.special.ndtr(z), "softplus": lambda: torch.logaddexp(z, torch.zeros_like(z))}[act]()


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "linear":
        y = _exact_act(s["x"].double() @ s["w"].double().t() + s["bias"].double(), case["act"])
        return {"y": y if s["residual"] is None else y + s["residual"].double()}
    if op == "linear_grad":
        dz = s["dy"].double()
        if s["pre"] is not None:
            z = s["pre"].double().requires_grad_()
            (dz,) = torch.autograd.grad(_exact_act(z, case["act"]), z, dz)
        return {"dx": dz @ s["w"].double(), "dw": dz.t() @ s["x"].double(), "dbias": dz.sum(0)}
    if op == "conv_step":
        z = s["bias"].double() + s["x"].double() * s["w"][:, -1].double()
        z = z + (s["state"].double() * s["w"][:, :-1].double().t()).sum(1)
        return {"y": z * torch.sigmoid(z), "state": torch.cat([s["state"][:, 1:], s["x"][:, None]], 1).double()}
    if op.startswith("conv"):
        got = _exact_conv(s, op == "conv_grad")
    elif op == "scan_step":
        s["lead"] = (case["batch"], 1)
        s.update({k: s[k][:, None] for k in ("x", "delta", "z", "B", "C")})
        got = _exact_scan(s, False)
        return {"y": got["y"], "state": got["state_out"]}
    else:
        got = _exact_scan(s, op == "scan_grad")
    like = {"y": "x", "dx": "x", "ddelta": "x", "dz": "x", "dB": "B", "dC": "C"}
    return {k: v.reshape(s[like[k]].shape) if k in like else v for k, v in got.items()}
