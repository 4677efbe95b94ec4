"""Binding with stream=: what a call allocates for itself belongs to that stream, on which the kernels write it, and is initialised there.  No GPU: the
library and torch's stream context are stand-ins that record."""
import contextlib

import pytest
import torch

bf16 = torch.bfloat16


class Side:
    cuda_stream = 1234


class Recorder:
    def __init__(self):
        self.active, self.allocated, self.launched, self.lent = [None], [], [], 0


@pytest.fixture
def rec(monkeypatch):
    from paper_2405_17991_b200 import binding as b
    r = Recorder()

    @contextlib.contextmanager
    def stream_context(s):
        r.active.append(s)
        yield
        r.active.pop()

    def recording(make):
        def call(*args, **kw):
            r.allocated.append(r.active[-1])
            return make(*args, **kw)
        return call

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name == "velora_workspace_bytes":
                    return 512
                r.launched.append((name, args[-1]))
                return 0
            return call

    def lend(t):
        r.lent += 1

    monkeypatch.setattr(torch.cuda, "stream", stream_context)
    for name in ("empty", "empty_strided", "empty_like", "zeros"):
        monkeypatch.setattr(torch, name, recording(getattr(torch, name)))
    monkeypatch.setattr(b, "lib", lambda: Library())
    monkeypatch.setattr(b, "_mat", lambda t, name: (t.data_ptr(), t.stride(0)))
    monkeypatch.setattr(b, "_vec", lambda t: t.data_ptr())
    monkeypatch.setattr(b, "_tokens", lambda t, n, dtype, name: t.data_ptr())
    monkeypatch.setattr(b, "_here", lambda *t: None)
    monkeypatch.setattr(b, "_lend", lend, raising=False)
    monkeypatch.setattr(b, "_stream", lambda s: (s or r.active[-1]).cuda_stream if s or r.active[-1] else 0)
    return r


N, D, O, DSUB = 4, 64, 24, 8
X, dY, W = (torch.ones(s, dtype=bf16) for s in ((N, D), (N, O), (O, D)))
Z, v, P, a = torch.ones((N, 8)), torch.ones(DSUB), torch.ones((O, 8)), torch.ones(DSUB)
Q, E = torch.ones((N, D), dtype=torch.int8), torch.ones((N, 2), dtype=torch.uint8)
t, lse = torch.ones(N, dtype=torch.int64), torch.ones(N)
# (call, tensors that it returns and made itself)
CALLS = {
    "velora_init_v": (lambda f, s: f(X, DSUB, stream=s), 1),
    "velora_compress": (lambda f, s: f(X, v, stream=s), 1),
    "velora_reconstruct": (lambda f, s: f(Z, v, D, stream=s), 1),
    "velora_weight_grad": (lambda f, s: f(dY, Z, v, D, stream=s), 1),
    "velora_linear_forward": (lambda f, s: f(X, W, v, stream=s), 2),
    "velora_linear_backward": (lambda f, s: f(dY, W, Z, v, stream=s), 2),
    "velora_dense_product": (lambda f, s: f(0, X, W, stream=s), 1),
    "velora_z8_calibrate": (lambda f, s: f(X, v, stream=s), 3),
    "velora_subtoken_sum": (lambda f, s: f(X, DSUB, stream=s), 1),
    "velora_update_v": (lambda f, s: f(X, DSUB, 0.5, a, v, stream=s), 0),
    "velora_normalize_v": (lambda f, s: f(a, stream=s), 1),
    "velora_weight_grad_p": (lambda f, s: f(dY, Z, D, DSUB, stream=s), 1),
    "velora_expand_p": (lambda f, s: f(P, v, D, stream=s), 1),
    "velora_checkpoint_store": (lambda f, s: f(X, stream=s), 2),
    "velora_checkpoint_load": (lambda f, s: f(Q, E, stream=s), 1),
    "velora_checkpoint_weight_grad": (lambda f, s: f(dY, Q, E, stream=s), 1),
    "velora_head_loss": (lambda f, s: f(X, W, t, stream=s), 2),
    "velora_head_loss_backward": (lambda f, s: f(X, W, t, lse, lse, stream=s), 2),
}


def test_every_call_with_a_stream_is_here():
    import inspect

    from paper_2405_17991_b200 import binding as b
    takes = {n for n, f in vars(b).items() if n.startswith("velora_") and callable(f) and "stream" in inspect.signature(f).parameters}
    # these allocate nothing, or are the allocation itself
    assert takes - set(CALLS) == {"velora_workspace_alloc", "velora_workspace_init", "velora_workspace_status", "velora_device_error",
                                  "velora_selftest_wait_timeout", "velora_init_v_static", "velora_linear_step_host"}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_allocations_belong_to_the_stream(rec, name):
    from paper_2405_17991_b200 import binding as b
    call, made = CALLS[name]
    side = Side()
    call(getattr(b, name), side)
    assert rec.active == [None]
    assert len(rec.allocated) >= made and all(s is side for s in rec.allocated)
    assert rec.launched[-1] == (name, 1234) and all(s == 1234 for _, s in rec.launched)
    assert rec.lent == made                                    # the caller's own stream may still read them when they are let go


def test_workspace_for_a_stream(rec):
    from paper_2405_17991_b200 import binding as b
    side = Side()
    b.velora_workspace_alloc(512, "cpu", side)
    assert rec.allocated == [side] and rec.launched == [("velora_workspace_init", 1234)]
    b.velora_workspace_alloc(512, "cpu")
    assert rec.allocated == [side, None] and rec.launched[-1] == ("velora_workspace_init", 0)
