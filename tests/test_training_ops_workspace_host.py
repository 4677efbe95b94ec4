"""CPU-only: a workspace that is no memory of the current device, or not in one piece, is refused before anything is launched."""
import pytest
import torch


@pytest.fixture
def b(monkeypatch):
    from paper_2405_17991_b200 import binding

    class Library:
        def __getattr__(self, name):
            def call(*args):
                raise AssertionError("reached %s" % name)
            return call

    monkeypatch.setattr(binding, "lib", lambda: Library())
    monkeypatch.setattr(binding, "_mat", lambda t, name: (t.data_ptr(), t.stride(0)))
    monkeypatch.setattr(binding, "_tokens", lambda t, n, dtype, name: t.data_ptr())
    monkeypatch.setattr(binding, "_stream", lambda s: 0)
    monkeypatch.setattr(binding, "_raw_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    return binding


class OnCard(torch.Tensor):
    """A tensor that says it is on device 0."""
    def get_device(self):
        return 0


def card(t):
    return t.as_subclass(OnCard)


CALLS = ["checkpoint_weight_grad", "head_loss", "head_loss_backward"]


def call(b, name, ws):
    X, W, t = card(torch.ones((4, 64), dtype=torch.bfloat16)), card(torch.ones((24, 64), dtype=torch.bfloat16)), card(torch.ones(4, dtype=torch.int64))
    f = lambda: card(torch.ones(4))  # noqa: E731
    if name == "checkpoint_weight_grad":
        return b.velora_checkpoint_weight_grad(card(torch.ones((4, 24), dtype=torch.bfloat16)), card(torch.ones((4, 64), dtype=torch.int8)),
                                               card(torch.ones((4, 2), dtype=torch.uint8)), dW=card(torch.empty_like(W)), ws=ws)
    if name == "head_loss":
        return b.velora_head_loss(X, W, t, loss=f(), lse=f(), ws=ws)
    return b.velora_head_loss_backward(X, W, t, f(), f(), dX=card(torch.empty_like(X)), dW=card(torch.empty_like(W)), ws=ws)


@pytest.mark.parametrize("name", CALLS)
def test_workspace_of_another_device(b, name):
    with pytest.raises(ValueError, match="current device"):
        call(b, name, torch.zeros(1 << 16, dtype=torch.uint8))


@pytest.mark.parametrize("name", CALLS)
def test_workspace_in_pieces(b, name):
    with pytest.raises(ValueError, match="contiguous"):
        call(b, name, card(torch.zeros(16, dtype=torch.uint8).expand(1 << 12, 16)))


@pytest.mark.parametrize("name", CALLS)
def test_workspace_that_is_taken(b, name):
    with pytest.raises(AssertionError, match="reached velora_" + name):
        call(b, name, card(torch.zeros(1 << 16, dtype=torch.uint8)))
