"""Linear attention where its chunks' tables, exponents and 16-bit operands have their limits, against the 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2603_09221_b200 import block
from tests import attention_util as au

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, H, F = torch.bfloat16, torch.float16, torch.float32


def _inputs(tokens, heads, dk, dv, dtype, seed, groups=None):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s, t=dtype: torch.randn(s, generator=g, device=DEV).to(t)  # noqa: E731
    return dict(q=r(1, tokens, groups or heads, dk), k=r(1, tokens, groups or heads, dk), v=r(1, tokens, heads, dv), A=-torch.rand(heads, generator=g, device=DEV) * 0.2 - 0.01,
                delta=r(1, tokens, heads).abs(), state=r(1, heads, dk, dv, t=F), dy=r(1, tokens, heads, dv), dlast=r(1, heads, dk, dv, t=F))


def _forward(i, scale=None):
    last = torch.empty_like(i["state"])
    return block.decay_attention(i["q"], i["k"], i["v"], i["A"], i["delta"], scale=scale, state=i["state"], state_out=last), last


def _grads(i, scale=None, **kw):
    return block.decay_attention_grad(i["dy"], i["q"], i["k"], i["v"], i["A"], i["delta"], scale=scale, state=i["state"], dstate_out=i["dlast"], **kw)


@pytest.mark.parametrize("dtype", [B, H])
def test_tables_of_many_chunks_are_whole(dtype):
    """Chunks whose decays differ, in walks that load the next ones meanwhile: the same bits every time."""
    i = _inputs(5000, 2, 64, 64, dtype, 3)
    i["delta"][:, ::3] = 0.01
    (y, last), grads = _forward(i), _grads(i)
    for _ in range(30):
        (y2, last2), got = _forward(i), _grads(i)
        assert torch.equal(y, y2) and torch.equal(last, last2) and all(torch.equal(got[n], grads[n]) for n in grads)
    assert block.device_error(0) == 0
