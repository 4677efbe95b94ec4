"""Distillation at temperatures that are no powers of two, teachers' logits at the ends of their type, small workspaces of few fp32 tokens: against the
definition in 64 bits, with the bounds of test_gpu_head_distill where no others are given."""
import pytest
import torch

from test_gpu_head_confident import SureReference, check_rows, sure_batch
from test_gpu_head_distill import U, Reference, backward, batch, check, forward, guard, half_step, vl  # noqa: F401

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("t_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("K", [5, 64, 300])
@pytest.mark.parametrize("N", [12, 150])
def test_logits_at_the_ends_of_their_type(vl, N, K, t_dtype, whole):  # noqa: F811
    """Finite logits whose quotient by T is not.  Compared with logits that mean the same: only differences count where nothing is given, and beside a given
    log sum a share is zero."""
    p = batch(N, 64, 900, K, torch.bfloat16, N + K, 0.25, "none", False, t_dtype)
    p["i"] = p["i"].abs() % 900
    low, high, inf = torch.finfo(t_dtype).min, torch.finfo(t_dtype).max, float("inf")
    q = {**p, "t": p["t"].clone()}
    p["t"][0::6], q["t"][0::6] = low, (-1000.0 if whole else 0.0)                          # all alike
    p["t"][1::6, 1:], q["t"][1::6, 1:] = low, -inf                                          # one counts
    p["t"][2::6, :2], q["t"][2::6, :2] = low, (-1000.0 if whole else 0.0)                  # two, and the others have no share
    p["t"][2::6, 2:] = q["t"][2::6, 2:] = -inf
    p["t"][3::6] = q["t"][3::6] = -inf                                                      # none
    if whole:
        p["lse"] = q["lse"] = torch.full((N,), 60.0, device=DEV)
    else:
        p["t"][4::6], q["t"][4::6] = 1.0, -inf                                              # one has it all
        p["t"][4::6, K // 2], q["t"][4::6, K // 2] = high, 0.0
    ref = Reference(q)
    loss, lse = forward(vl, p)
    check(loss, ref.loss, ref.loss_bound, "loss")
    check(lse, ref.lse, ref.lse_bound, "lse")
    dX, dW = backward(vl, p, lse)
    check(dX, ref.dX, ref.dX_bound, "dX", half_step(torch.bfloat16))
    check(dW, ref.dW, ref.dW_bound, "dW", half_step(torch.bfloat16))
