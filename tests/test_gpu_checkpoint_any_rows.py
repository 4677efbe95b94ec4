"""The weight gradient from 8-bit checkpoints of a bf16 dY whose rows start anywhere: the product on the tensor cores, from a packed copy."""
import pytest
import torch

from _util import Guard
from test_gpu_checkpoint import DEV, finite_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vl():
    import paper_2405_17991_b200 as pkg
    pkg.lib()
    return pkg


@pytest.mark.parametrize("left,right", [(1, 0), (0, 5), (5, 2)])
@pytest.mark.parametrize("N,D,O", [(520, 264, 2056), (2000, 512, 1376), (300, 77, 45)])
def test_same_bits_as_aligned_rows(vl, N, D, O, left, right):
    """fp32 results: the CUDA cores round their sums, the tensor cores truncate, so equal bits are those of one product."""
    X, dY = finite_inputs(N, D, O, torch.bfloat16, N + O)
    aligned = torch.zeros((N, -(-O // 8) * 8), device=DEV, dtype=torch.bfloat16)[:, :O]
    aligned.copy_(dY)
    moved = torch.full((N, left + O + right), 7.0, device=DEV, dtype=torch.bfloat16)[:, left:left + O]
    moved.copy_(dY)
    assert moved.data_ptr() % 16 or moved.stride(0) % 8
    Q, E = vl.velora_checkpoint_store(X)
    guard, out = Guard(DEV), []
    for y, any_rows in ((aligned, False), (moved, True)):
        dW = guard.mat(O, D, torch.float32)
        ws = guard.workspace(vl, vl.velora_workspace_bytes(vl.OP_CHECKPOINT_WEIGHT_GRAD, N, D, O, 1, any_rows))
        vl.velora_checkpoint_weight_grad(y, Q, E, dW, ws=ws)
        assert vl.velora_workspace_status(ws) == 0
        out.append(dW)
    assert torch.equal(*out)
    assert torch.equal(out[0], vl.velora_checkpoint_weight_grad(moved, Q, E, dw_dtype=torch.float32, dW=guard.mat(O, D, torch.float32)))
    guard.check()
