"""What selective scans and their gradients keep over long sequences in float32: every output within a bound that is carried along
with the recurrences (scan_bounds.py: it forgets what the state forgets), and small in the 2-norm.

The 2-norm.  The mean error of the exponentials of decays that last, at most 1.2e-8, adds up over a memory of 200 tokens to 2.4e-6; what is random in a token's
decay, product and sums is below 2^-22 and adds up in squares, 14 times that, 3.4e-6; sums over states and channels by less.  1e-5 is
allowed to what holds a state or a co-state, twice that to what holds both."""
import numpy as np
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import block_util as bu
from tests import scan_bounds as sb
from tests.test_scan_bounds import inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = torch.float32
BOTH = ("ddelta", "dA", "ddelta_bias")


def _values(lead, d, n, groups, slow, cuts=None, gated=True, seed=7):
    """Arguments of the calls, and the same in 64 bits for the plain forms."""
    rng = np.random.default_rng(seed)
    rows = int(np.prod(lead))
    v = inputs(rng, rows, d, n, groups, slow, gated)
    seqs = bu.spans(lead, cuts)
    v["state"], v["seqs"] = rng.standard_normal((len(seqs), d, n)).astype(np.float32), seqs
    more = dict(dy=rng.standard_normal((rows, d)).astype(np.float32), dlast=rng.standard_normal((len(seqs), d, n)).astype(np.float32))
    put = lambda a, rowwise: torch.from_numpy(a).to(DEV).reshape(*((*lead, *a.shape[1:]) if rowwise else a.shape))  # noqa: E731
    args = {k: None if v[k] is None else put(v[k], k in ("x", "delta", "B", "C", "z")) for k in ("x", "delta", "A", "B", "C", "D", "z", "delta_bias", "state")}
    args["offsets"] = None if cuts is None else torch.tensor(cuts, dtype=torch.int32, device=DEV)
    plain = {k: a.astype(np.float64) if isinstance(a, np.ndarray) else a for k, a in v.items()}
    return dict(args, softplus=True), plain, {k: put(a, k == "dy") for k, a in more.items()}, {k: a.astype(np.float64) for k, a in more.items()}


def _hold(got, want, bound, limit, what):
    keep = ~np.isnan(want).reshape(want.shape[0], -1).any(1)
    have = got.reshape(want.shape)[torch.from_numpy(keep).to(DEV)]
    bu.within(have, want[keep], bound[keep], F, what)
    off = np.linalg.norm(bu.f64(have) - want[keep]) / np.linalg.norm(want[keep])
    assert off <= limit, (what, off)


def _check_forward(args, plain, y, last, piece):
    (want, states, _), (ey, el) = bu.scan(**plain), sb.forward(**plain, piece=piece)
    _hold(y, want, ey, 1e-5, "y")
    _hold(last, states, el, 1e-5, "state_out")


CASES = [((1, 1025), 8, 16, 1, None), ((2, 700), 3, 4, 1, None), ((1, 513), 40, 64, 2, None), ((1, 4000), 24, 16, 3, None),
         ((1310,), 8, 16, 1, [0, 0, 5, 400, 400, 1300, 1301, 1301]), ((2000,), 24, 32, 2, [3, 1500, 1997]), ((2, 300), 130, 16, 1, None)]


@pytest.mark.parametrize("slow", [False, True])
@pytest.mark.parametrize("lead, d, n, groups, cuts", CASES)
def test_prompts_and_gradients(lead, d, n, groups, cuts, slow):
    args, plain, more, more64 = _values(lead, d, n, groups, slow, cuts)
    last = torch.empty_like(args["state"])
    y = block.selective_scan(**args, state_out=last)
    _check_forward(args, plain, y, last, 128)                        # (few channels: pieces of 128 tokens, the shortest there are)
    got = block.selective_scan_grad(more["dy"], **args, dstate_out=more["dlast"])
    want, bound = bu.scan_grad(**plain, **more64), sb.gradients(**plain, **more64, piece=16)
    for k in want:
        _hold(got[k], want[k], bound[k], 2e-5 if k in BOTH else 1e-5, k)


@pytest.mark.parametrize("slow", [False, True])
def test_single_tokens_one_behind_the_other(slow):
    args, plain, _, _ = _values((1, 600), 40, 16, 2, slow)
    state = args.pop("state").clone()
    args.pop("offsets")
    rows = ("x", "delta", "B", "C", "z")
    ys = [block.selective_scan_step(**{k: v[:, t] if k in rows else v for k, v in args.items()}, state=state) for t in range(600)]
    _check_forward(args, plain, torch.stack(ys, 1), state, 1)


def test_a_prompt_in_calls_of_odd_lengths():
    args, plain, _, _ = _values((2, 900), 16, 16, 1, True)
    state, rows, ys, at = args.pop("state").clone(), ("x", "delta", "B", "C", "z"), [], 0
    for length in (1, 299, 7, 512, 81):
        part = {k: v[:, at:at + length] if k in rows else v for k, v in args.items()}
        ys.append(block.selective_scan(**part, state=state, state_out=state))
        at += length
    _check_forward(args, plain, torch.cat(ys, 1), state, 128)
