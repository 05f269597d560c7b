"""Calls at the edges of what include/ttc_block.h allows: no rows with outputs in place."""
import pytest
import torch

from paper_2603_09221_b200 import block

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
