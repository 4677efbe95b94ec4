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


@pytest.mark.parametrize("T", [1.0, 1.1, 1.5, 2.5, 5.0, 0.7])
@pytest.mark.parametrize("N", [10, 100, 300])
def test_one_column_has_the_whole_share(vl, N, T):  # noqa: F811
    """G = g / T (exp(l / T - lse) - 1) would be zero, and shows what the two passes' l / T and lse differ by.  That is lse's rounding to fp32, u |lse|, and
    2^-20 for an exponential in each pass (2^-22) and the
    roundings of products and sums near one behind them: a temperature is no source of its own."""
    g = torch.Generator(device=DEV).manual_seed(N)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    D = 64
    p = {"X": (100 * r(N, D)).bfloat16(), "W": r(1, D).bfloat16(), "i": torch.zeros((N, 1), dtype=torch.int64, device=DEV), "t": r(N, 1), "lse": None,
         "g": torch.ones(N, device=DEV), "T": T}
    loss, lse = forward(vl, p)
    dX, _ = backward(vl, p, lse, need_dW=False)
    bound = (U * lse.double().abs() + 2.0 ** -20)[:, None] / T * p["W"].double().abs() * (1 + 2.0 ** -6)          # two roundings to bf16
    worst = (dX.double().abs() / bound).max().item()
    assert worst <= 1.0, worst


@pytest.mark.parametrize("T", [1.1, 2.5])
@pytest.mark.parametrize("N", [4, 100, 300])
def test_a_student_that_agrees_at_another_temperature(vl, N, T):  # noqa: F811
    D, V = 256, 600
    p = batch(N, D, V, V, torch.bfloat16, 33, T)
    l = p["X"].double() @ p["W"].double().t()
    p["i"] = torch.stack([torch.randperm(V, device=DEV) for _ in range(N)])
    p["t"] = l.gather(1, p["i"]).float()
    ref = Reference(p)
    loss, lse = forward(vl, p)
    check(loss, ref.loss, ref.loss_bound, "loss")
    dX, dW = backward(vl, p, lse)
    check(dX, ref.dX, ref.dX_bound, "dX", half_step(torch.bfloat16))
    check(dW, ref.dW, ref.dW_bound, "dW", half_step(torch.bfloat16))
    q = torch.softmax(l / T, 1)
    assert dX.double().norm() <= 2.0 ** -12 / T * ((q * p["g"].double()[:, None].abs()) @ p["W"].double().abs()).norm()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1.5, 0.7])
@pytest.mark.parametrize("N", [8, 100, 300])
def test_gradients_of_sure_tokens_at_another_temperature(vl, N, T, dtype):  # noqa: F811
    """Logits over T as in test_gpu_head_confident; its reference takes W / T for W."""
    D, V = 2048, 2000
    X, W, t, dloss = sure_batch(N, D, V, dtype, False, N + D)
    X = (X.double() * T).to(dtype)
    ref = SureReference(X, W.double() / T, t, dloss, N)
    p = {"X": X, "W": W, "i": t[:, None].contiguous(), "t": torch.zeros((N, 1), device=DEV), "lse": None, "g": dloss, "T": T}
    loss, lse = forward(vl, p)
    dX, dW = backward(vl, p, lse)
    check_rows(dX, ref.dX, ref.dX_bound, "dX")
    hit = torch.unique(t)
    check_rows(dW[hit], ref.dW[hit] / T, ref.dW_bound[hit] / T, "dW")


@pytest.mark.parametrize("T", [1.0, 1.1, 1.5, 2.5, 5.0, 0.7])
@pytest.mark.parametrize("N", [10, 100, 300])
def test_one_column_in_fp32(vl, N, T):  # noqa: F811
    """A logit over T is rounded once, to the same number in both passes, and is lse here: exp(0) - 1 is zero."""
    g = torch.Generator(device=DEV).manual_seed(N)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    D = 64
    p = {"X": 100 * r(N, D), "W": r(1, D), "i": torch.zeros((N, 1), dtype=torch.int64, device=DEV), "t": r(N, 1), "lse": None,
         "g": torch.ones(N, device=DEV), "T": T}
    loss, lse = forward(vl, p)
    dX, _ = backward(vl, p, lse, need_dW=False)
    assert not dX.any() and not loss.any()


@pytest.mark.parametrize("dw_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1.5, 3.0, 6.0, 256 / 257])
def test_a_temperature_is_not_rounded_into_every_gradient(vl, T, dw_dtype):  # noqa: F811
    """bf16, more than 64 tokens, each with one entry that the student knows nothing of: G at the entries is -g / T (1 - q), q below 2^-10.  1 / T rounded to bf16 in
    all of them would be off by up to 2^-8, always the same way; without that factor they are within q of -g, g equal for all.  The other
    columns' q g round by 2^-8 of themselves, N / V of them to an entry, so that they are 2^-5 of dW in norm at the most.  Then the output's own rounding:
    bf16's root mean square of 1.66e-3 and a tenth more."""
    N, D, V = 512, 256, 4096
    g = torch.Generator(device=DEV).manual_seed(7)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    p = {"X": r(N, D).bfloat16(), "W": (0.002 * r(V, D)).bfloat16(), "i": torch.randint(V, (N, 1), generator=g, device=DEV), "t": r(N, 1), "lse": None,
         "g": torch.full((N,), T * T / N, device=DEV), "T": T}
    _, lse = forward(vl, p)
    x, w = p["X"].double(), p["W"].double()
    q = torch.softmax(x @ w.t() / T, 1)
    assert q.max() < 2.0 ** -10
    G = q.clone().scatter_add_(1, p["i"], torch.full((N, 1), -1.0, device=DEV, dtype=torch.float64)) * (T / N)
    dX, dW = backward(vl, p, lse, dw_dtype=dw_dtype)
    own = {torch.bfloat16: 1.83e-3, torch.float32: 0.0}
    for got, ref, rounding in ((dX, G @ w, own[torch.bfloat16]), (dW, G.t() @ x, own[dw_dtype])):
        bound = ((2.0 ** -10 + 2.0 ** -13) ** 2 + rounding ** 2) ** 0.5
        error = ((got.double() - ref).norm() / ref.norm()).item()
        assert error <= bound, error


@pytest.mark.parametrize("N", [1, 5, 16])
@pytest.mark.parametrize("D,V", [(200, 700), (203, 1000), (4099, 520)])
def test_few_fp32_tokens_in_a_small_workspace(vl, guard, N, D, V):  # noqa: F811
    """Room for one sum of dX instead of its slices, and for a piece of 256 columns: what every piece gives is added to that one."""
    p = batch(N, D, V, 3, torch.float32, N + D, 1.5, "some" if N > 4 else "none", True)
    ref = Reference(p)
    _, lse = forward(vl, p)
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    slices = min(256, 1184 // -(-D // 512))
    one, pitch = N * (-(-D // 8) * 8), up(V)
    front = vl.velora_workspace_bytes(vl.OP_HEAD_DISTILL_BACKWARD | vl.OP_F32, N, D, V, 3, False) - up(4 * N * pitch)
    least = front - up(4 * one * slices) + up(4 * one)
    for room in (256, 512):
        dX, dW = backward(vl, p, lse, ws=guard.workspace(vl, least + 4 * N * room))
        check(dX, ref.dX, ref.dX_bound, "dX")
        check(dW, ref.dW, ref.dW_bound, "dW")
    with pytest.raises(vl.VeloraError):
        backward(vl, p, lse, ws=guard.workspace(vl, least + 4 * N * 256 - 1))
