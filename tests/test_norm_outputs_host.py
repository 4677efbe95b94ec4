"""CPU-only checks of where a layer norm's outputs may lie, with stand-ins for the library: see test_norm_distill_host.py."""
import pytest
import torch

from test_norm_distill_host import D, N, each, seen, w  # noqa: F401


def test_a_norm_in_place_returns_no_rows_for_the_backward_pass(seen):  # noqa: F811
    from paper_2405_17991_b200 import training_ops as t
    X = torch.ones((N, D), dtype=torch.bfloat16)
    Y = torch.ones_like(X)
    assert t.velora_layer_norm(X, w)[1] is X and t.velora_layer_norm(X, w, Y=Y)[1] is X
    for same in (X, X[:], X.view(N, D)):
        Y, H, mean, rstd = t.velora_layer_norm(X, w, Y=same)
        assert Y is same and H is None
        with pytest.raises(ValueError, match="H is None"):
            t.velora_layer_norm_backward(X, H, mean, rstd, w)
    R = torch.ones_like(X)
    assert t.velora_layer_norm(X, w, residual=R, Y=X)[1] is not None
    assert t.velora_layer_norm(X, w, residual=R, Y=R, H=X)[1] is X


def test_one_address_for_h_and_y_is_refused():
    from paper_2405_17991_b200 import binding, build
    from test_norm_distill_host import P, norm
    build.build()
    f = norm(binding)
    assert f() == f(R=P(0)) == f(H=P(0x20000), Y=P(0x20000)) == binding.ERR_INVALID_ARG
