"""CPU-only checks of the layer norm and of distillation into a linear head: refusals from metadata alone, workspace sizes, whose stream allocations are."""
import contextlib
import ctypes

import pytest
import torch

P = ctypes.c_void_p
good, odd, null = P(0x10000), P(0x10001), P(0)
BIG = 1 << 34


@pytest.fixture(scope="module")
def b():
    from paper_2405_17991_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def caller(f, defaults):
    return lambda **k: f(*[k.get(n, d) for n, d in defaults])


def norm(b):
    return caller(b.lib().velora_layer_norm, [("X", good), ("ldx", 64), ("R", good), ("ldr", 64), ("w", good), ("b", good), ("pt", b.F32), ("eps", 1e-5),
                                              ("H", good), ("ldh", 64), ("Y", good), ("ldy", 64), ("mean", good), ("rstd", good), ("dt", b.BF16),
                                              ("N", 4), ("D", 64), ("s", null)])


def norm_backward(b):
    return caller(b.lib().velora_layer_norm_backward, [("dY", good), ("lddy", 64), ("H", good), ("ldh", 64), ("mean", good), ("rstd", good), ("w", good),
                                                       ("pt", b.F32), ("dH", good), ("lddh", 64), ("dX", good), ("lddx", 64), ("dw", good), ("db", good),
                                                       ("dwt", b.F32), ("beta", 0), ("dt", b.BF16), ("N", 4), ("D", 64), ("ws", good), ("n", BIG),
                                                       ("s", null)])


LISTS = [("X", good), ("ldx", 64), ("W", good), ("ldw", 64), ("i", good), ("ldi", 8), ("t", good), ("tt", 0), ("ldt", 8), ("tl", null), ("T", 2.0), ("K", 8)]


def distill(b):
    return caller(b.lib().velora_head_distill, LISTS + [("loss", good), ("lse", good), ("dt", b.BF16), ("N", 4), ("D", 64), ("V", 100), ("ws", good),
                                                        ("n", BIG), ("s", null)])


def distill_backward(b):
    return caller(b.lib().velora_head_distill_backward,
                  LISTS + [("lse", good), ("g", good), ("dX", good), ("lddx", 64), ("dW", good), ("dwt", b.BF16), ("lddw", 64), ("beta", 0), ("dt", b.BF16),
                           ("N", 4), ("D", 64), ("V", 100), ("ws", good), ("n", BIG), ("s", null)])


def test_norm_refusals(b):
    f = norm(b)
    for name in ("X", "Y"):
        assert f(**{name: null}) == b.ERR_INVALID_ARG, name
    for name in ("ldx", "ldr", "ldh", "ldy"):
        assert f(**{name: 63}) == b.ERR_INVALID_ARG, name
    for name in ("X", "R", "H", "Y", "w", "b", "mean", "rstd"):
        assert f(**{name: odd}) == b.ERR_ALIGNMENT, name
    for eps in (-1e-5, float("nan"), float("inf"), -float("inf")):
        assert f(eps=eps) == b.ERR_INVALID_ARG
    assert f(N=-1) == b.ERR_INVALID_ARG
    assert f(D=0) == b.ERR_INVALID_ARG
    assert f(D=(1 << 30) + 1) == b.ERR_UNSUPPORTED
    assert f(N=(1 << 40) + 1) == b.ERR_UNSUPPORTED
    assert f(dt=b.FP8_E4M3) == b.ERR_UNSUPPORTED
    assert f(pt=b.FP8_E4M3) == b.ERR_UNSUPPORTED
    assert f(N=0, X=null, Y=null, pt=7, w=null, b=null) == b.OK


def test_norm_backward_refusals(b):
    f = norm_backward(b)
    for name in ("dY", "H", "mean", "rstd"):
        assert f(**{name: null}) == b.ERR_INVALID_ARG, name
    for name in ("lddy", "ldh", "lddh", "lddx"):
        assert f(**{name: 63}) == b.ERR_INVALID_ARG, name
    for name in ("dY", "H", "mean", "rstd", "w", "dH", "dX", "dw", "db"):
        assert f(**{name: odd}) == b.ERR_ALIGNMENT, name
    assert f(beta=2) == b.ERR_INVALID_ARG
    assert f(N=-1) == b.ERR_INVALID_ARG
    assert f(D=0) == b.ERR_INVALID_ARG
    assert f(D=(1 << 30) + 1) == b.ERR_UNSUPPORTED
    assert f(dt=5) == b.ERR_UNSUPPORTED
    assert f(dwt=b.FP8_E4M3) == b.ERR_UNSUPPORTED
    assert f(ws=null) == b.ERR_WORKSPACE
    assert f(n=256 + 2 * 4 * 64 * 4 - 1) == b.ERR_WORKSPACE
    assert f(ws=P(0x10008)) == b.ERR_ALIGNMENT
    assert f(dX=null, dw=null, db=null, ws=null) == b.OK                # nothing is asked for
    assert f(N=0, beta=1, dY=null, ws=null) == b.OK


def test_distill_refusals(b):
    F, B = distill(b), distill_backward(b)
    for f in (F, B):
        for name in ("X", "W", "i", "t", "lse"):
            assert f(**{name: null}) == b.ERR_INVALID_ARG, name
        for name, v in (("ldx", 63), ("ldw", 63), ("ldi", 7), ("ldt", 7), ("N", -1), ("D", 0), ("V", 0), ("K", 0), ("K", -3)):
            assert f(**{name: v}) == b.ERR_INVALID_ARG, name
        for T in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
            assert f(T=T) == b.ERR_INVALID_ARG, T
        assert f(K=1025, ldi=1025, ldt=1025) == b.ERR_UNSUPPORTED
        for name in ("N", "V"):
            assert f(**{name: (1 << 30) + 1}) == b.ERR_UNSUPPORTED
        assert f(dt=b.FP8_E4M3) == b.ERR_UNSUPPORTED
        assert f(tt=b.FP8_E4M3) == b.ERR_UNSUPPORTED
        for name in ("X", "W", "t", "tl", "lse"):
            assert f(**{name: P(0x10001)}) == b.ERR_ALIGNMENT, name
        assert f(i=P(0x10004)) == b.ERR_ALIGNMENT
        assert f(ws=null) == b.ERR_WORKSPACE
        assert f(n=1024) == b.ERR_WORKSPACE
        assert f(ws=P(0x10008)) == b.ERR_ALIGNMENT
    assert F(loss=null) == b.ERR_INVALID_ARG
    assert F(N=0, X=null, i=null, t=null, loss=null) == b.OK
    assert B(g=null) == b.ERR_INVALID_ARG
    assert B(lddx=63) == b.ERR_INVALID_ARG
    assert B(lddw=63) == b.ERR_INVALID_ARG
    assert B(beta=2) == b.ERR_INVALID_ARG
    assert B(dwt=b.FP8_E4M3) == b.ERR_UNSUPPORTED
    assert B(dX=odd) == b.ERR_ALIGNMENT
    assert B(dX=null, dW=null) == b.OK
    assert B(N=0, beta=1, X=null) == b.OK


def test_workspace_sizes(b):
    size = b.lib().velora_workspace_bytes
    for op, like in ((b.OP_HEAD_DISTILL, b.OP_HEAD_LOSS), (b.OP_HEAD_DISTILL_BACKWARD, b.OP_HEAD_LOSS_BACKWARD)):
        for flags in (0, b.OP_F32, b.OP_ANY_ROWS, b.OP_F32 | b.OP_ANY_ROWS):
            assert size(op | flags, 100, 64, 1000, 128) >= size(like | flags, 100, 64, 1000, 1) + 100 * 128 * 8      # K may be more than D
        assert size(op, 0, 64, 1000, 8) >= 256
        assert size(op, 100, 64, 1000, 1024) > size(op, 100, 64, 1000, 1)
        for bad in ((100, 64, 0, 8), (-1, 64, 1000, 8), (100, 0, 1000, 8), (100, 64, 1000, 0), (100, 64, 1000, 1025)):
            assert size(op, *bad) == 0
        assert size(op | 1024, 100, 64, 1000, 8) == 0
    N, D, V = 8192, 4096, 128000                          # neither the logits of a whole vocabulary nor their gradients
    assert size(b.OP_HEAD_DISTILL, N, D, V, 64) < N * V
    assert size(b.OP_HEAD_DISTILL_BACKWARD, N, D, V, 64) < N * V
    op = b.OP_LAYER_NORM_BACKWARD
    assert size(op, 4, 64, 1, 1) == size(op | b.OP_F32, 4, 64, 1, 1) >= 256 + 2 * 4 * 64 * 4
    assert size(op, 1 << 40, 64, 1, 1) == size(op, 1 << 20, 64, 1, 1)
    assert size(op, 0, 64, 1, 1) >= 256
    assert size(op, -1, 64, 1, 1) == 0 and size(op, 4, 0, 1, 1) == 0


def test_binding_refuses(b):
    import paper_2405_17991_b200 as vl
    X = torch.zeros((4, 64), dtype=torch.bfloat16)
    i, t = torch.zeros((4, 8), dtype=torch.int64), torch.zeros((4, 8))
    for call in (lambda: vl.velora_layer_norm(X), lambda: vl.velora_layer_norm(X[0]), lambda: vl.velora_layer_norm_backward(X, X, X, X),
                 lambda: vl.velora_head_distill(X, X, i, t), lambda: vl.velora_head_distill(X, X, i[:3], t[:3]),
                 lambda: vl.velora_head_distill(X, X, i, t[:, :7]), lambda: vl.velora_head_distill(X, X, i.int(), t),
                 lambda: vl.velora_head_distill_backward(X, X, i, t, t[0], t[0])):
        with pytest.raises(ValueError):                       # no CUDA tensor, or of the wrong shape
            call()
    assert b.velora_layer_norm is vl.velora_layer_norm
    with pytest.raises(AttributeError):
        b.velora_no_such_call


# ---- the binding with stand-ins for the library and torch's streams: see test_streams_host.py ----
N, D, V, K = 4, 64, 24, 8
X, W, R = (torch.ones((N, D), dtype=torch.bfloat16) for _ in range(3))
W = torch.ones((V, D), dtype=torch.bfloat16)
w = torch.ones(D)
index, logits, each = torch.ones((N, K), dtype=torch.int64), torch.ones((N, K)), torch.ones(N)
# (call, tensors that it returns and has made itself)
CALLS = {
    "velora_layer_norm": (lambda f, **k: f(X, w, w, residual=R, **k), 4),
    "velora_layer_norm_backward": (lambda f, **k: f(X, X, each, each, w, **k), 3),
    "velora_head_distill": (lambda f, **k: f(X, W, index, logits, **k), 2),
    "velora_head_distill_backward": (lambda f, **k: f(X, W, index, logits, each, each, **k), 2),
}


class Side:
    cuda_stream = 1234


class Seen:
    def __init__(self):
        self.active, self.allocated, self.launched, self.lent = [None], [], [], 0


@pytest.fixture
def seen(monkeypatch):
    from paper_2405_17991_b200 import binding as b
    r = Seen()

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
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, recording(getattr(torch, name)))
    monkeypatch.setattr(b, "lib", lambda: Library())
    monkeypatch.setattr(b, "_mat", lambda t, name: (t.data_ptr(), t.stride(0)))
    monkeypatch.setattr(b, "_tokens", lambda t, n, dtype, name: t.data_ptr())
    monkeypatch.setattr(b, "_here", lambda *t: None)
    monkeypatch.setattr(b, "_lend", lend)
    monkeypatch.setattr(b, "_stream", lambda s: (s or r.active[-1]).cuda_stream if s or r.active[-1] else 0)
    from paper_2405_17991_b200 import training_ops
    monkeypatch.setattr(training_ops, "_columns", lambda t, d, name: None if t is None else t.data_ptr())
    return r


@pytest.mark.parametrize("name", sorted(CALLS))
def test_allocations_belong_to_the_stream(seen, name):
    from paper_2405_17991_b200 import training_ops
    call, made = CALLS[name]
    side = Side()
    call(getattr(training_ops, name), stream=side)
    assert seen.active == [None]
    assert len(seen.allocated) >= made and all(s is side for s in seen.allocated)
    assert seen.launched[-1] == (name, 1234) and all(s == 1234 for _, s in seen.launched)
    assert seen.lent == made                                  # the caller's own stream may still read them when they are let go


@pytest.mark.parametrize("name", sorted(set(CALLS) - {"velora_layer_norm"}))
def test_workspaces_that_are_refused(seen, monkeypatch, name):
    from paper_2405_17991_b200 import binding as b, training_ops
    call, _ = CALLS[name]
    with pytest.raises(ValueError, match="contiguous"):
        call(getattr(training_ops, name), ws=torch.zeros(16, dtype=torch.uint8).expand(1 << 12, 16))
    monkeypatch.undo()
    monkeypatch.setattr(b, "_mat", lambda t, name: (t.data_ptr(), t.stride(0)))
    monkeypatch.setattr(b, "_tokens", lambda t, n, dtype, name: t.data_ptr())
    monkeypatch.setattr(training_ops, "_columns", lambda t, d, name: None if t is None else t.data_ptr())
    monkeypatch.setattr(b, "_raw_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    with pytest.raises(ValueError, match="current device"):    # tensors on the host
        call(getattr(training_ops, name), ws=torch.zeros(1 << 16, dtype=torch.uint8))
