"""CPU-only checks of the 8-bit checkpoints and the loss of a linear head: refusals from metadata alone and workspace sizes."""
import ctypes

import pytest

P = ctypes.c_void_p
good, odd, null = P(0x10000), P(0x10001), P(0)


@pytest.fixture(scope="module")
def b():
    from paper_2405_17991_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def test_checkpoint_refusals(b):
    st, ld, wg = b.lib().velora_checkpoint_store, b.lib().velora_checkpoint_load, b.lib().velora_checkpoint_weight_grad
    assert st(good, b.BF16, -1, 64, 64, good, 64, good, 2, null) == b.ERR_INVALID_ARG
    assert st(good, b.BF16, 4, 0, 64, good, 64, good, 2, null) == b.ERR_INVALID_ARG
    assert st(null, b.BF16, 4, 64, 64, good, 64, good, 2, null) == b.ERR_INVALID_ARG
    assert st(good, b.BF16, 4, 64, 64, null, 64, good, 2, null) == b.ERR_INVALID_ARG
    assert st(good, b.BF16, 4, 64, 64, good, 64, null, 2, null) == b.ERR_INVALID_ARG
    assert st(good, b.BF16, 4, 64, 63, good, 64, good, 2, null) == b.ERR_INVALID_ARG
    assert st(good, b.BF16, 4, 64, 64, good, 63, good, 2, null) == b.ERR_INVALID_ARG
    assert st(good, b.BF16, 4, 65, 65, good, 65, good, 2, null) == b.ERR_INVALID_ARG            # 65 columns are 3 blocks
    assert st(good, b.FP8_E4M3, 4, 64, 64, good, 64, good, 2, null) == b.ERR_UNSUPPORTED
    assert st(good, b.BF16, 4, 1 << 31, 1 << 31, good, 1 << 31, good, 1 << 31, null) == b.ERR_UNSUPPORTED
    assert st(odd, b.BF16, 4, 64, 64, good, 64, good, 2, null) == b.ERR_ALIGNMENT
    assert st(null, b.BF16, 0, 64, 64, null, 64, null, 2, null) == b.OK
    assert ld(good, 64, good, 2, 4, 64, null, b.BF16, 64, null) == b.ERR_INVALID_ARG
    assert ld(good, 64, good, 2, 4, 64, good, b.BF16, 63, null) == b.ERR_INVALID_ARG
    assert ld(good, 64, good, 1, 4, 64, good, b.BF16, 64, null) == b.ERR_INVALID_ARG
    assert ld(good, 64, good, 2, 4, 64, good, 9, 64, null) == b.ERR_UNSUPPORTED
    assert ld(good, 64, good, 2, 4, 64, odd, b.F32, 64, null) == b.ERR_ALIGNMENT
    assert ld(null, 64, null, 2, 0, 64, null, b.BF16, 64, null) == b.OK
    big = 1 << 30
    args = lambda **k: [k.get(n, d) for n, d in (("dY", good), ("dt", b.BF16), ("N", 4), ("O", 8), ("lddy", 8), ("Q", good), ("ldq", 64), ("E", good),   # noqa: E731
                                                 ("lde", 2), ("D", 64), ("dW", good), ("dwt", b.BF16), ("lddw", 64), ("beta", 0), ("ws", good), ("n", big), ("s", null))]
    assert wg(*args(dY=null)) == b.ERR_INVALID_ARG
    assert wg(*args(O=0)) == b.ERR_INVALID_ARG
    assert wg(*args(lddy=7)) == b.ERR_INVALID_ARG
    assert wg(*args(lddw=63)) == b.ERR_INVALID_ARG
    assert wg(*args(beta=2)) == b.ERR_INVALID_ARG
    assert wg(*args(dW=null)) == b.ERR_INVALID_ARG
    assert wg(*args(Q=null)) == b.ERR_INVALID_ARG
    assert wg(*args(lde=1)) == b.ERR_INVALID_ARG
    assert wg(*args(dwt=b.FP8_E4M3)) == b.ERR_UNSUPPORTED
    assert wg(*args(dt=5)) == b.ERR_UNSUPPORTED
    assert wg(*args(dW=odd)) == b.ERR_ALIGNMENT
    assert wg(*args(ws=null)) == b.ERR_WORKSPACE
    assert wg(*args(n=255)) == b.ERR_WORKSPACE
    assert wg(*args(ws=P(0x10008))) == b.ERR_ALIGNMENT
    assert wg(*args(N=0, dY=null, Q=null, E=null, beta=1)) == b.OK


def test_head_refusals(b):
    fw, bw = b.lib().velora_head_loss, b.lib().velora_head_loss_backward
    big = 1 << 34
    F = lambda **k: fw(*[k.get(n, d) for n, d in (("X", good), ("ldx", 64), ("W", good), ("ldw", 64), ("t", good), ("loss", good), ("lse", good),   # noqa: E731
                                                 ("dt", b.BF16), ("N", 4), ("D", 64), ("V", 100), ("ws", good), ("n", big), ("s", null))])
    B = lambda **k: bw(*[k.get(n, d) for n, d in (("X", good), ("ldx", 64), ("W", good), ("ldw", 64), ("t", good), ("lse", good), ("g", good),   # noqa: E731
                                                 ("dX", good), ("lddx", 64), ("dW", good), ("dwt", b.BF16), ("lddw", 64), ("beta", 0),
                                                 ("dt", b.BF16), ("N", 4), ("D", 64), ("V", 100), ("ws", good), ("n", big), ("s", null))])
    for f in (F, B):
        for name in ("X", "W", "t", "lse"):
            assert f(**{name: null}) == b.ERR_INVALID_ARG, name
        for name, v in (("ldx", 63), ("ldw", 63), ("N", -1), ("D", 0), ("V", 0)):
            assert f(**{name: v}) == b.ERR_INVALID_ARG, name
        for name in ("N", "V"):
            assert f(**{name: (1 << 30) + 1}) == b.ERR_UNSUPPORTED
        assert f(N=1 << 29, V=1 << 29) == b.ERR_UNSUPPORTED
        assert f(dt=b.FP8_E4M3) == b.ERR_UNSUPPORTED
        assert f(X=odd) == b.ERR_ALIGNMENT
        assert f(t=P(0x10004)) == b.ERR_ALIGNMENT
        assert f(lse=P(0x10002)) == b.ERR_ALIGNMENT
        assert f(ws=null) == b.ERR_WORKSPACE
        assert f(n=1024) == b.ERR_WORKSPACE
        assert f(ws=P(0x10008)) == b.ERR_ALIGNMENT
    assert F(loss=null) == b.ERR_INVALID_ARG
    assert F(N=0, X=null, t=null, loss=null) == b.OK
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
    for op in (b.OP_HEAD_LOSS, b.OP_HEAD_LOSS_BACKWARD, b.OP_CHECKPOINT_WEIGHT_GRAD):
        assert size(op, 100, 64, 1000, 1) >= 256
        assert size(op, 0, 64, 1000, 1) >= 256
        assert size(op, 100, 64, 0, 1) == 0
        assert size(op, -1, 64, 1000, 1) == 0
    # neither the logits of a whole vocabulary nor their gradients
    N, D, V = 8192, 4096, 128000
    assert size(b.OP_HEAD_LOSS, N, D, V, 1) < N * V
    assert size(b.OP_HEAD_LOSS_BACKWARD, N, D, V, 1) < N * V
    assert size(b.OP_HEAD_LOSS_BACKWARD | b.OP_F32, N, D, V, 1) < 2 * N * V


def test_binding_refuses_shapes(b):
    import torch
    X = torch.zeros((4, 64), dtype=torch.bfloat16)
    for call in (lambda: b.velora_checkpoint_store(X), lambda: b.velora_head_loss(X, X, torch.zeros(4, dtype=torch.int64)),
                 lambda: b.velora_checkpoint_load(torch.zeros((4, 64), dtype=torch.int8), torch.zeros((4, 1), dtype=torch.uint8))):
        with pytest.raises(ValueError):                       # no CUDA tensor, or of the wrong shape
            call()
    with pytest.raises(ValueError):
        b.velora_checkpoint_load(torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8))


def test_binding_refuses_tensors_of_another_device(b, monkeypatch):
    """The kernels go to the current device's stream: a tensor of another device is refused before anything is launched."""
    import torch

    class Elsewhere:
        device = "cuda:7"

        def get_device(self):
            return 7

    monkeypatch.setattr(b, "_raw_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    with pytest.raises(ValueError, match="current device"):
        b._here(Elsewhere())
