"""Layer norms whose outputs lie on their inputs, rows of one very large value, fp32 rows around the longest that a backward pass with dH holds: against the
formula in 64 bits, with the bounds of test_gpu_layer_norm."""
import pytest
import torch

from test_gpu_layer_norm import EPS, Backward, Forward, batch, check, guard, half_step, run, vl  # noqa: F401

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D", [(40, 768), (40, 1001), (3, 16400)])
def test_a_norm_in_place_leaves_nothing_for_the_backward_pass(vl, N, D, dtype):  # noqa: F811
    """Y on X, nothing added: H would be X, which holds Y by then."""
    p = batch(N, D, dtype, 10)
    Y, H, mean, rstd = vl.velora_layer_norm(p["X"], p["w"], p["b"])
    assert H is p["X"]
    want = vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, p["w"])
    for same in (lambda X: X, lambda X: X[:], lambda X: X.view(N, D)):
        X = p["X"].clone()
        at, gone, m, r = vl.velora_layer_norm(X, p["w"], p["b"], Y=same(X))
        assert gone is None and torch.equal(at, Y) and torch.equal(m, mean) and torch.equal(r, rstd)
        with pytest.raises(ValueError):
            vl.velora_layer_norm_backward(p["dY"], gone, m, r, p["w"])
    kept = p["X"].clone()                                     # what a caller does who wants both
    X = p["X"].clone()
    vl.velora_layer_norm(X, p["w"], p["b"], Y=X, mean=mean, rstd=rstd)
    assert all(torch.equal(x, y) for x, y in zip(vl.velora_layer_norm_backward(p["dY"], kept, mean, rstd, p["w"]), want))


@pytest.mark.parametrize("N,D", [(4, 64), (4, 1001)])
def test_one_address_for_h_and_y_is_refused(vl, N, D):  # noqa: F811
    p = batch(N, D, torch.bfloat16, 1)
    out = torch.full_like(p["X"], 3.0)
    for Y, H in ((out, out), (p["X"], p["X"]), (p["R"], p["R"])):
        with pytest.raises(vl.VeloraError):
            vl.velora_layer_norm(p["X"], p["w"], p["b"], residual=p["R"], Y=Y, H=H)
    assert bool((out == 3.0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,power,eps", [(65, 120, EPS), (100, 120, EPS), (250, 120, EPS), (513, 110, 1e-12), (1001, 110, 1e-12), (2050, 110, 1e-12), (5461, 110, 1e-12), (9001, 110, 1e-12)])
def test_rows_of_one_very_large_value(vl, D, power, eps, dtype):  # noqa: F811
    """xhat is zero, although the mean times 1 / sqrt(eps) is beyond fp32: nothing of that may come in from columns that a thread does not have."""
    g = torch.Generator(device=DEV).manual_seed(D)
    X = torch.full((6, D), 2.0 ** power, device=DEV).to(dtype)
    X[3:] *= -1
    dY = torch.randn((6, D), generator=g, device=DEV).to(dtype)
    dH = torch.randn((6, D), generator=g, device=DEV).to(dtype)
    w, b = 1 + 0.3 * torch.randn(D, generator=g, device=DEV), torch.randn(D, generator=g, device=DEV)
    Y, H, mean, rstd = vl.velora_layer_norm(X, w, b, eps)
    assert torch.equal(mean, X[:, 0].float()) and bool((mean.abs().double() * rstd.double() > 3.5e38).all())
    ref = Forward(X, None, w, b, eps)
    check(Y, ref.Y, ref.Y_bound, "Y", half_step(dtype))
    for more in (None, dH):
        back = Backward(dY, X, mean, rstd, w, more)
        dX, dw, db = vl.velora_layer_norm_backward(dY, H, mean, rstd, w, dH=more)
        check(dX, back.dX, back.dX_bound, "dX", half_step(dtype))
        check(dw, back.dw, back.dw_bound, "dweight")
        check(db, back.db, back.db_bound, "dbias")


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("D", [9209, 9211, 9213, 9217, 10239, 12285, 12287])
def test_fp32_rows_around_the_longest_that_are_held(vl, guard, D, residual):  # noqa: F811
    run(vl, guard, batch(300, D, torch.float32, D), residual, torch.float32, ld=D)
