"""Linear attention with a decay for each head, and the norms around a block with its gate and residual scale, as cases that can
be timed and compared: forward, backward and, where a model decodes, for single tokens.

``run`` computes a case in its plain form, in elementary torch operations in 32 bits, or, where ``own`` is true, by the
calls of ``paper_2603_09221_b200.block`` that a program makes.  Notation: sequences of equal length, or packed one behind the
other with ``offsets``; ``heads`` heads of ``dv`` value channels, ``groups`` groups of them that share queries and keys of
``dk`` channels; ``d`` channels of the residual stream.

  attend       D_t = softplus(delta_t + bias), or 1;  S_t = exp(A D_t) S_{t-1} + k_t v_t';  y_t = q_t S_t / sqrt(dk),
               the state S in front of a sequence given, the last one returned
  norm         u = x rms(x) w_post  (in groups);  u = u silu(z);  h = r + s u;  y = h rms(h) w_pre,
               rms(v) = 1 / sqrt(mean(v^2) + eps);  any of the parts may be missing
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CHUNK = 64                      # tokens that the plain form takes together
EPS = 1e-6


def _attend(op, batch, tokens, heads, groups, dk, dv, dtype, decay="token", packed=False, name=None):
    c = dict(op=op, batch=batch, tokens=tokens, heads=heads, groups=groups, dk=dk, dv=dv, dtype=dtype, decay=decay)
    if op != "attend_step":
        c.update(packed=packed)
    return c if name is None else dict(c, name=name)


def _norm(op, rows, d, dtype, post=0, gate=False, scale=False, residual=False, pre=True, name=None):
    c = dict(op=op, rows=rows, d=d, dtype=dtype, post=post, gate=gate, scale=scale, residual=residual, pre=pre)
    return c if name is None else dict(c, name=name)


def listed():
    # `tokens` counts the tokens of all sequences together where they are packed, else those of one sequence.
    return [
        # Prompts of 2048 tokens, 4 sequences, 16 heads.
        _attend("attend", 4, 2048, 16, 16, 128, 128, "bf16", name="attend_prompt"),
        # One long prompt of odd length with small heads, whose decays are fixed.
        _attend("attend", 1, 16381, 8, 8, 64, 64, "f16", decay="head", name="attend_long"),
        # Packed documents; eight heads to each set of queries and keys.
        _attend("attend", 7, 4093, 16, 2, 64, 128, "bf16", packed=True, name="attend_packed"),
        # A few tokens behind a prompt, heads of odd widths.
        _attend("attend", 3, 29, 6, 3, 36, 20, "bf16", name="attend_few_tokens"),
        # Decoding: one new token of each of 64 sequences; the states are 268 MB, read and written.
        _attend("attend_step", 64, 1, 16, 16, 128, 128, "bf16", name="attend_decode"),
        # Decoding a single sequence.
        _attend("attend_step", 1, 1, 16, 16, 64, 64, "f16", decay="head", name="attend_decode_one"),
        # Training: every gradient of 4 sequences of 1024 tokens.
        _attend("attend_grad", 4, 1024, 16, 16, 128, 128, "bf16", name="attend_train"),
        # Training on 11 documents of different lengths packed into 8191 rows, two heads to each set of queries and keys.
        _attend("attend_grad", 11, 8191, 8, 4, 64, 64, "f16", packed=True, name="attend_train_packed"),
        # Decoding: the residual stream of 8 sequences moves on, and is normed for the next block.
        _norm("norm", 8, 2048, "bf16", residual=True, name="norm_decode"),
        # Prompts: everything between two blocks, the block's output normed for each of 32 heads and gated.
        _norm("norm", 8192, 4096, "bf16", post=32, gate=True, scale=True, residual=True, name="norm_block"),
        # Training: the gradients of the same over 4 sequences of 2048 tokens.
        _norm("norm_grad", 8192, 2048, "bf16", post=16, gate=True, scale=True, residual=True, name="norm_train"),
        # Training in float32 on packed rows of an odd number: the gated norm of 8 heads of 125 channels alone.
        _norm("norm_grad", 4093, 1000, "f32", post=8, gate=True, pre=False, name="norm_train_heads"),
    ]


def _spread(rng, low, high):
    """A whole number between the two, evenly over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(("attend", "attend", "attend_step", "attend_grad", "norm", "norm_grad"))
    if op.startswith("norm"):
        d = _spread(rng, 64, 4096)
        d = d if rng.random() < 0.3 else -(-d // 64) * 64
        most = 8192 * 4096 if op == "norm" else 8192 * 2048                                    # no more than the largest listed
        rows = min(most // d, _spread(rng, 1, 32768))
        post = rng.choice([0] + [g for g in (1, 2, 4, 8, 16, 32) if d % g == 0 and d // g >= 16])
        residual = rng.random() < 0.6
        pre = post == 0 or rng.random() < 0.7
        return _norm(op, rows, d, rng.choice(("bf16", "bf16", "f16", "f32")), post, rng.random() < 0.5, rng.random() < 0.4, residual, pre)
    dtype, decay = rng.choice(("bf16", "bf16", "f16")), rng.choice(("token", "token", "head"))
    dk, dv = _spread(rng, 16, 128), _spread(rng, 16, 128)
    if rng.random() < 0.6:                                      # widths of heads are multiples of 16; odd ones are served too
        dk, dv = -(-dk // 16) * 16, -(-dv // 16) * 16
    groups = rng.choice((1, 2, 4, 8, 16))
    heads = groups * rng.choice([r for r in (1, 1, 2, 4, 8) if r * groups <= 16])
    if op == "attend_step":
        return _attend(op, _spread(rng, 1, 64), 1, heads, groups, dk, dv, dtype, decay)
    most = (4 * 2048 * 16 if op == "attend" else 4 * 1024 * 16) // heads
    rows = _spread(rng, 16, min(most, 16384))
    batch, packed = min(rows, _spread(rng, 1, 16)), rng.random() < 0.4
    return _attend(op, batch, rows if packed else max(1, rows // batch), heads, groups, dk, dv, dtype, decay, packed)


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
    if op.startswith("norm"):
        rows, d = case["rows"], case["d"]
        weight = lambda have, at=1.0: at + randn(d, scale=0.1 * at, dtype=torch.float32) if have else None  # noqa: E731
        s.update(x=randn(rows, d, scale=1.5), w_post=weight(case["post"]), z=randn(rows, d) if case["gate"] else None,
                 scale=weight(case["scale"], 0.3), w_pre=weight(case["pre"]))
        if op == "norm":
            s["residual"] = randn(rows, d, scale=2.0) if case["residual"] else None
        else:
            changed = case["post"] or case["gate"] or case["scale"] or case["residual"]
            s["h"] = randn(rows, d, scale=2.0) if changed else None                             # as the forward call wrote it
            s["dh"] = randn(rows, d) if changed else None
            s["dy"] = randn(rows, d) if case["pre"] else None
        return s
    batch, heads, groups, dk, dv = (case[k] for k in ("batch", "heads", "groups", "dk", "dv"))
    packed = case.get("packed", False)
    rows = case["tokens"] if packed else batch * case["tokens"]
    lead = (rows,) if packed else (batch,) if op == "attend_step" else (batch, case["tokens"])
    s["lead"] = lead
    s["offsets"] = _offsets(gen, batch, rows) if packed else None
    # the lengths, as the program that packed the rows knows them
    s["lengths"] = s["offsets"].diff().tolist() if packed else [1 if op == "attend_step" else case["tokens"]] * batch
    s.update(q=randn(*lead, groups, dk), k=randn(*lead, groups, dk), v=randn(*lead, heads, dv),
             state=randn(batch, heads, dk, dv, scale=0.3, dtype=torch.float32), delta=None, delta_bias=None)
    if case["decay"] == "token":
        # decay rates 1 .. 16, step sizes between 1e-3 and 1e-1 (softplus of what a projection gives plus a bias)
        step = torch.exp(torch.rand(heads, generator=gen, device=DEVICE) * math.log(100.0) + math.log(1e-3))
        s.update(A=-(1 + 15 * torch.rand(heads, generator=gen, device=DEVICE)), delta_bias=step + torch.log(-torch.expm1(-step)),
                 delta=randn(*lead, heads, scale=0.5))
    else:
        # the heads remember 8 to 1024 tokens
        s["A"] = -torch.exp(-math.log(2.0) * (3 + 7 * torch.rand(heads, generator=gen, device=DEVICE)))
    if op == "attend_grad":
        s.update(dy=randn(*lead, heads, dv), dstate_out=randn(batch, heads, dk, dv, dtype=torch.float32))
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _softplus(z):
    return z.clamp(min=0) + torch.log1p(torch.exp(-z.abs()))


def _silu(z):
    return z / (1 + torch.exp(-z))


def _steps(s):
    """Step sizes D and their slopes, [*lead, heads] in 32 bits."""
    if s["delta"] is None:
        one = torch.ones((*s["lead"], s["case"]["heads"]), device=DEVICE)
        return one, one
    raw = s["delta"].float() + s["delta_bias"]
    return _softplus(raw), 1 / (1 + torch.exp(-raw))


def _wide(v, heads):
    """[.., groups, dk] -> [.., heads, dk]: the group of every head."""
    return v.float().repeat_interleave(heads // v.shape[-2], -2)


class _Chunks:
    """Rows in chunks: [*lead, heads, c] <-> [chunks, batch, heads, CHUNK, c] in 32 bits, zeros behind a sequence's end."""

    def __init__(self, s):
        self.s, self.lengths = s, s["lengths"]
        self.n = max(1, -(-max(self.lengths) // CHUNK))
        at = torch.arange(self.n * CHUNK, device=DEVICE)
        length = torch.tensor(self.lengths, device=DEVICE)
        self.batch = len(self.lengths)
        first = torch.cumsum(length, 0) - length
        self.inside = at[None] < length[:, None]                                               # [batch, places]
        self.row = torch.where(self.inside, first[:, None] + at[None], 0)

    def split(self, v):
        v = v.float().flatten(0, len(self.s["lead"]) - 1)
        if v.shape[0] == 0:
            v = v.new_zeros((1, *v.shape[1:]))
        v = torch.where(self.inside[..., None, None], v[self.row], 0.0)
        return v.reshape(self.batch, self.n, CHUNK, *v.shape[2:]).permute(1, 0, 3, 2, 4)

    def join(self, v):
        v = v.permute(1, 0, 3, 2, 4).reshape(self.batch, self.n * CHUNK, v.shape[2], v.shape[4])
        return v[self.inside].reshape(*self.s["lead"], *v.shape[2:])


def _decays(c, steps, A):
    """Within the chunks, sums of log decays in 64 bits: exp(G_i - G_j) for j <= i, exp(G_i), exp(G_C - G_j), exp(G_C)."""
    G = torch.cumsum((c.split(steps[..., None])[..., 0] * A[:, None]).double(), -1)
    below = torch.ones((CHUNK, CHUNK), dtype=torch.bool, device=DEVICE).tril()
    pair = torch.where(below, torch.exp(torch.where(below, G[..., :, None] - G[..., None, :], 0.0)), 0.0).float()
    return pair, torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None], torch.exp(G[..., -1]).float()[..., None, None]


def _states(first, decay, added):
    """The state in front of every chunk, and the one behind the last."""
    states, S = [], first
    for i in range(added.shape[0]):
        states.append(S)
        S = decay[i] * S + added[i]
    return torch.stack(states), S


def _plain_attend(s):
    heads, t = s["case"]["heads"], s["v"].dtype
    c = _Chunks(s)
    q, k, v = c.split(_wide(s["q"], heads)) * s["case"]["dk"] ** -0.5, c.split(_wide(s["k"], heads)), c.split(s["v"])
    pair, front, back, whole = _decays(c, _steps(s)[0], s["A"])
    S, last = _states(s["state"], whole, (k * back).transpose(-1, -2) @ v)
    y = ((q @ k.transpose(-1, -2)) * pair) @ v + front * (q @ S)
    return {"y": c.join(y).to(t), "state_out": last}


def _plain_attend_step(s):
    heads = s["case"]["heads"]
    q, k = _wide(s["q"], heads) * s["case"]["dk"] ** -0.5, _wide(s["k"], heads)
    decay = torch.exp(_steps(s)[0] * s["A"])
    s["state"].mul_(decay[..., None, None]).add_(k[..., None] * s["v"].float()[..., None, :])
    return {"y": (q[..., None] * s["state"]).sum(-2).to(s["v"].dtype), "state": s["state"]}


def _plain_attend_grad(s):
    case, t = s["case"], s["v"].dtype
    heads, groups, scale = case["heads"], case["groups"], case["dk"] ** -0.5
    c = _Chunks(s)
    q, k, v, dy = c.split(_wide(s["q"], heads)) * scale, c.split(_wide(s["k"], heads)), c.split(s["v"]), c.split(s["dy"])
    steps, slopes = _steps(s)
    pair, front, back, whole = _decays(c, steps, s["A"])
    S, _ = _states(s["state"], whole, (k * back).transpose(-1, -2) @ v)
    Z, dstate = _states(s["dstate_out"], whole.flip(0), ((q * front).transpose(-1, -2) @ dy).flip(0))
    Z = Z.flip(0)
    score, slope = (q @ k.transpose(-1, -2)) * pair, dy @ v.transpose(-1, -2)
    far_q, far_k = front * (dy @ S.transpose(-1, -2)), back * (v @ Z.transpose(-1, -2))
    dq = scale * ((slope * pair) @ k + far_q)
    dk = (slope * pair).transpose(-1, -2) @ q + far_k
    dv = score.transpose(-1, -2) @ dy + back * (k @ Z)
    # log decays: what lies on both sides of a token, in 64 bits since large sums cancel
    both = (score * slope).double().tril(-1)
    later = (q * far_q).double().sum(-1) + both.sum(-1) - both.sum(-2)
    earlier = (k * far_k).double().sum(-1)
    dl = later.flip(-1).cumsum(-1).flip(-1) + earlier.cumsum(-1) - earlier + (whole.double() * Z * S).sum((-1, -2))[..., None]
    dl = c.join(dl.float()[..., None])[..., 0]
    share = lambda g: c.join(g).unflatten(-2, (groups, heads // groups)).sum(-2).to(t)  # noqa: E731
    got = {"dq": share(dq), "dk": share(dk), "dv": c.join(dv).to(t), "dA": (dl * steps).flatten(0, -2).double().sum(0).float(), "dstate": dstate}
    if s["delta"] is not None:
        ddelta = dl * s["A"] * slopes
        got.update(ddelta=ddelta.to(t), ddelta_bias=ddelta.flatten(0, -2).double().sum(0).float())
    return got


def _rms(v, groups=1):
    """1 / sqrt(mean of squares + eps) of every group of channels, spread over its channels."""
    size = v.shape[-1] // groups
    return (v.unflatten(-1, (groups, size)).square().mean(-1) + EPS).rsqrt().repeat_interleave(size, -1)


def _plain_norm(s):
    case, t = s["case"], s["x"].dtype
    u = s["x"].float()
    if case["post"]:
        u = u * _rms(u, case["post"]) * s["w_post"]
    if case["gate"]:
        u = u * _silu(s["z"].float())
    if case["scale"]:
        u = u * s["scale"]
    if case["residual"]:
        u = u + s["residual"].float()
    got = {"h": u.to(t)} if case["post"] or case["gate"] or case["scale"] or case["residual"] else {}
    if case["pre"]:
        got["y"] = (u * _rms(u) * s["w_pre"]).to(t)
    return got


def _back_through_norm(dy, v, w, groups=1):
    """Gradients with respect to v and w of v rms(v) w."""
    size, r = v.shape[-1] // groups, _rms(v, groups)
    n, g = v * r, dy * w
    mean = (n * g).unflatten(-1, (groups, size)).mean(-1).repeat_interleave(size, -1)
    return r * (g - n * mean), (dy * n).sum(0)


def _plain_norm_grad(s):
    case, t = s["case"], s["x"].dtype
    x = s["x"].float()
    dh, got = 0.0, {}
    if s["dh"] is not None:
        dh = s["dh"].float()
    if case["pre"]:
        from_y, got["dw_pre"] = _back_through_norm(s["dy"].float(), s["h"].float() if s["h"] is not None else x, s["w_pre"])
        dh = dh + from_y
    if case["residual"]:
        got["dresidual"] = dh.to(t)
    u = x * _rms(x, case["post"]) * s["w_post"] if case["post"] else x
    gate = _silu(s["z"].float()) if case["gate"] else 1.0
    if case["scale"]:
        got["dscale"] = (dh * u * gate).sum(0)
        dh = dh * s["scale"]
    if case["gate"]:
        z = s["z"].float()
        p = 1 / (1 + torch.exp(-z))
        got["dz"] = (dh * u * p * (1 + z * (1 - p))).to(t)
        dh = dh * gate
    if case["post"]:
        dh, got["dw_post"] = _back_through_norm(dh, x, s["w_post"], case["post"])
    got["dx"] = dh.to(t)
    return got


PLAIN = {"attend": _plain_attend, "attend_step": _plain_attend_step, "attend_grad": _plain_attend_grad, "norm": _plain_norm,
         "norm_grad": _plain_norm_grad}


# ---- the framework's calls --------------------------------------------------------------------------------------------

def _own(s):
    from paper_2603_09221_b200 import block
    case, op = s["case"], s["case"]["op"]
    if op == "norm":
        h, y = block.block_norm(s["x"], w_post=s["w_post"], z=s["z"], scale=s["scale"], residual=s["residual"], w_pre=s["w_pre"], eps=EPS,
                                groups=case["post"] or 1)
        got = {"h": h} if case["post"] or case["gate"] or case["scale"] or case["residual"] else {}
        return got if y is None else dict(got, y=y)
    if op == "norm_grad":
        return block.block_norm_grad(s["x"], h=s["h"], dy=s["dy"], dh=s["dh"], w_post=s["w_post"], z=s["z"], scale=s["scale"], w_pre=s["w_pre"], eps=EPS,
                                     groups=case["post"] or 1, residual=case["residual"])
    args = (s["q"], s["k"], s["v"], s["A"])
    more = dict(delta=s["delta"], delta_bias=s["delta_bias"], softplus=s["delta"] is not None, state=s["state"])
    if op == "attend":
        state_out = torch.empty_like(s["state"])
        return {"y": block.decay_attention(*args, **more, offsets=s["offsets"], state_out=state_out), "state_out": state_out}
    if op == "attend_step":
        return {"y": block.decay_attention_step(*args, **more), "state": s["state"]}
    return block.decay_attention_grad(s["dy"], *args, **more, offsets=s["offsets"], dstate_out=s["dstate_out"])


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    op, size = case["op"], 4 if case["dtype"] == "f32" else 2
    if op.startswith("norm"):
        n, changed = case["rows"] * case["d"], bool(case["post"] or case["gate"] or case["scale"] or case["residual"])
        vectors = 4 * case["d"] * (bool(case["post"]) + case["scale"] + case["pre"])
        if op == "norm":
            return {"bytes": size * n * (1 + case["gate"] + case["residual"] + changed + case["pre"]) + vectors, "flops": 15 * n}
        return {"bytes": size * n * (2 + 2 * case["gate"] + 2 * changed - (changed and not case["pre"]) + case["pre"] + case["residual"]) + 2 * vectors,
                "flops": 30 * n}
    batch, heads, groups, dk, dv = (case[k] for k in ("batch", "heads", "groups", "dk", "dv"))
    rows = case["tokens"] if case.get("packed") else batch * case["tokens"]
    states, shared, values, steps = batch * heads * dk * dv * 4, rows * groups * dk * size, rows * heads * dv * size, rows * heads * size
    steps = steps if case["decay"] == "token" else 0
    if op == "attend_grad":
        return {"bytes": 4 * shared + 3 * values + 2 * steps + 3 * states, "flops": 15 * rows * heads * dk * dv}
    return {"bytes": 2 * shared + 2 * values + steps + 2 * states, "flops": 5 * rows * heads * dk * dv}


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------

def _exact_attend(s, grad):
    """Token by token, as the recurrence is written; equal sequences side by side."""
    case = s["case"]
    heads, groups, dk = case["heads"], case["groups"], case["dk"]
    A, even = s["A"].double(), s["offsets"] is None
    view = (lambda v: v.double()) if even else (lambda v: v.double()[None])
    q, k = (view(s[n])[:, :, torch.arange(heads, device=DEVICE) // (heads // groups)] for n in ("q", "k"))
    q = q / math.sqrt(dk)
    v = view(s["v"])
    if s["delta"] is not None:
        raw = view(s["delta"]) + s["delta_bias"].double()
        steps, slopes = torch.logaddexp(raw, torch.zeros_like(raw)), torch.sigmoid(raw)
    else:
        steps = slopes = torch.ones_like(v[..., 0])
    a = torch.exp(A * steps)[..., None, None]
    if even:
        spans = [(0, v.shape[1], slice(0, v.shape[0]))]
    else:
        o = s["offsets"].tolist()
        spans = [(o[i], o[i + 1], slice(i, i + 1)) for i in range(len(o) - 1)]
    y, last = torch.empty_like(v), s["state"].double().clone()
    kept = {}
    for lo, hi, who in spans:
        S = s["state"][who].double()
        for t in range(lo, hi):
            if grad:
                kept[t] = S                                                                    # the state in front of the token
            S = a[:, t] * S + k[:, t, :, :, None] * v[:, t, :, None, :]
            y[:, t] = (q[:, t, :, None, :] @ S)[:, :, 0]
        last[who] = S
    if not grad:
        return {"y": y.reshape(s["v"].shape), "state_out": last}
    dy = view(s["dy"])
    dq, dk_, dv, dl = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(v[..., 0])
    dstate = s["dstate_out"].double().clone()
    for lo, hi, who in spans:
        Z = s["dstate_out"][who].double()
        for t in range(hi - 1, lo - 1, -1):
            S = a[:, t] * kept[t] + k[:, t, :, :, None] * v[:, t, :, None, :]
            dq[:, t] = (S @ dy[:, t, :, :, None])[..., 0]
            Z = Z + q[:, t, :, :, None] * dy[:, t, :, None, :]
            dk_[:, t] = (Z @ v[:, t, :, :, None])[..., 0]
            dv[:, t] = (k[:, t, :, None, :] @ Z)[:, :, 0]
            Z = a[:, t] * Z
            dl[:, t] = (Z * kept.pop(t)).sum((-1, -2))
        dstate[who] = Z
    narrow = lambda g, n: g.unflatten(2, (groups, heads // groups)).sum(3).reshape(s[n].shape)  # noqa: E731
    got = {"dq": narrow(dq, "q") / math.sqrt(dk), "dk": narrow(dk_, "k"), "dv": dv.reshape(s["v"].shape), "dA": (dl * steps).sum((0, 1)), "dstate": dstate}
    if s["delta"] is not None:
        ddelta = dl * A * slopes
        got.update(ddelta=ddelta.reshape(s["delta"].shape), ddelta_bias=ddelta.sum((0, 1)))
    return got


def _exact_norm(case, x, w_post, z, scale, residual, w_pre):
    """h and y; the norms as quotients by a root of the mean square."""
    n, d = x.shape
    u = x
    if case["post"]:
        g = u.reshape(n, case["post"], -1)
        u = (g / torch.sqrt(g.pow(2).mean(-1, keepdim=True) + EPS)).reshape(n, d) * w_post
    if case["gate"]:
        u = u * z * torch.sigmoid(z)
    if case["scale"]:
        u = scale * u
    if case["residual"]:
        u = residual + u
    return u, w_pre * u / torch.sqrt(u.pow(2).mean(-1, keepdim=True) + EPS) if case["pre"] else None


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "attend_step":
        s.update({k: s[k][:, None] for k in ("q", "k", "v", "delta") if s[k] is not None}, lead=(case["batch"], 1))
        got = _exact_attend(s, False)
        return {"y": got["y"][:, 0], "state": got["state_out"]}
    if op.startswith("attend"):
        return _exact_attend(s, op == "attend_grad")
    f = {k: v.double().requires_grad_(op == "norm_grad") if torch.is_tensor(v) else None for k, v in s.items() if k != "case"}
    if op == "norm":
        h, y = _exact_norm(case, *(f[k] for k in ("x", "w_post", "z", "scale", "residual", "w_pre")))
        got = {"h": h} if s["residual"] is not None or case["post"] or case["gate"] or case["scale"] else {}
        return dict(got, y=y) if case["pre"] else got
    # h comes rounded, as the forward call wrote it: the norm in front of the next block is differentiated at that h
    plain, ends = s["h"] is None, {}
    dh = f["dh"].detach() if f["dh"] is not None else torch.zeros_like(f["x"])
    if case["pre"]:
        at = f["x"] if plain else f["h"]
        _, y = _exact_norm(dict(case, post=0, gate=False, scale=False, residual=False), at, None, None, None, None, f["w_pre"])
        from_y, ends["dw_pre"] = torch.autograd.grad(y, (at, f["w_pre"]), f["dy"].detach())
        dh = dh + from_y
    if case["residual"]:
        ends["dresidual"] = dh
    u, _ = _exact_norm(dict(case, residual=False, pre=False), f["x"], f["w_post"], f["z"], f["scale"], None, None)
    names = [n for n, have in (("x", True), ("z", case["gate"]), ("scale", case["scale"]), ("w_post", case["post"])) if have]
    if plain:
        return dict(ends, dx=dh)
    return dict(ends, **{"d" + n: g for n, g in zip(names, torch.autograd.grad(u, [f[n] for n in names], dh))})
