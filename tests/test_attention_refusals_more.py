"""More of what linear attention and the norms refuse (no GPU needed)."""
import pytest
import torch

from paper_2603_09221_b200 import block, lqr

P = 1 << 20                 # an address that is never read: every call here is refused or only sized
INVALID = -1


def _norm_grad_status(residual, h, dresidual):
    """Gradients of y = rms(h) h w_pre with h = x + residual, or x."""
    lib = block._load()
    a = block._NORM_ARGS.pack(64, 48, 1, 1, 1e-6, P, 0, residual, h, 0, 48, 0, 48, 48, 0, 0, 0, P)
    g = block._NORM_GRADS.pack(6 * P, 0, 8 * P, 0, dresidual, 48, 0, 48, 0, 48, 0, 0, P)
    return lib.ttc_block_norm_grad_workspace(0, a, g), lqr.load_library().ttc_lqr_last_error().decode()


def test_the_norm_behind_a_residual_wants_h():
    """Without h, x would stand in for x + residual."""
    assert _norm_grad_status(0, 0, 0)[0] > 0                                        # nothing changes x
    assert _norm_grad_status(0, 4 * P, 10 * P)[0] > 0
    for residual, dresidual in ((3 * P, 0), (0, 10 * P), (3 * P, 10 * P)):
        status, text = _norm_grad_status(residual, 0, dresidual)
        assert status == INVALID and "h" in text
    x, w = torch.zeros((4, 16), dtype=torch.bfloat16), torch.zeros(16)
    for want in (None, ["dx"], ["dw_pre"]):
        with pytest.raises(ValueError, match="residual wants h"):
            block.block_norm_grad(x, dy=x, w_pre=w, residual=True, want=want)


@pytest.mark.parametrize("heads, dv", [(0, 32), (4, 0)])
def test_no_heads_or_no_channels(heads, dv):
    q, v = torch.zeros((2, 8, 2, 16), dtype=torch.bfloat16), torch.zeros((2, 8, heads, dv), dtype=torch.bfloat16)
    A, state = torch.zeros(heads), torch.zeros((2, heads, 16, dv))
    for call in (lambda: block.decay_attention(q, q, v, A), lambda: block.decay_attention_grad(v, q, q, v, A), lambda: block.decay_attention_step(q[:, 0], q[:, 0], v[:, 0], A, state)):
        with pytest.raises(ValueError):
            call()
