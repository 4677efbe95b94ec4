"""The weight gradient from 8-bit checkpoints where the last wave of its tiles is cut over the contraction, against the definition and not against
what is read back."""
import pytest
import torch

from _util import C_SUM, TOL_GEMM, Guard, assert_matches
from test_gpu_checkpoint import DEV, definition, finite_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vl():
    import paper_2405_17991_b200 as pkg
    pkg.lib()
    return pkg


@pytest.fixture
def guard():
    g = Guard(DEV)
    yield g
    g.check()


@pytest.mark.parametrize("dw_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,O", [(8200, 2304, 2304), (8200, 2303, 2305), (9001, 4096, 1300)])
def test_cut_last_wave_against_the_definition(vl, guard, N, D, O, dw_dtype):
    X, dY = finite_inputs(N, D, O, torch.bfloat16, N + D + O + 1)
    Q, E = vl.velora_checkpoint_store(X)
    ref = dY.double().t() @ torch.from_numpy(definition(X)[2]).to(DEV)
    for again in range(3):                                     # whoever counts in last, the same bits
        dW = guard.mat(O, D, dw_dtype)
        vl.velora_checkpoint_weight_grad(dY, Q, E, dW)
        if again == 0:
            first = dW.clone()
            assert_matches(dW, ref.cpu().numpy(), TOL_GEMM, "dW", c=C_SUM)
        assert torch.equal(dW, first)
