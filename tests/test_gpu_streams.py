"""Calls on a stream that is not the current one, with memory of their own: nothing that the current stream allocates and writes meanwhile reaches
their results, nor the other way round."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def vl():
    import paper_2405_17991_b200 as pkg
    pkg.lib()
    return pkg


def operands(dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    N, D, O, V = 2100, 1024, 2304, 4001
    t = torch.where(torch.rand(N, generator=g, device=DEV) < 0.3, -1, torch.randint(V, (N,), generator=g, device=DEV))
    return r(N, D).to(dtype), r(N, O).to(dtype), (r(V, D) / D ** 0.5).to(dtype), t, r(N), r(O, D).to(dtype), r(16)


def calls(vl, X, dY, W, t, g, Wl, v, **kw):
    Q, E = vl.velora_checkpoint_store(X, **kw)
    dWq = vl.velora_checkpoint_weight_grad(dY, Q, E, **kw)
    loss, lse = vl.velora_head_loss(X, W, t, **kw)
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, g, **kw)
    Y, Z = vl.velora_linear_forward(X, Wl, v, **kw)
    dXl, dWl = vl.velora_linear_backward(dY, Wl, Z, v, **kw)
    return [dWq, loss, dX, dW, Y, dXl, dWl, vl.velora_checkpoint_load(Q, E, **kw)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_memory_of_calls_on_another_stream(vl, dtype):
    ops = operands(dtype)
    want = [x.clone() for x in calls(vl, *ops)]
    other = torch.cuda.Stream()
    for _ in range(3):
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            torch.cuda._sleep(20_000_000)                     # some 10 ms: the calls' kernels are behind it
        got = calls(vl, *ops, stream=other)
        mine = []
        for _ in range(40):                                    # whatever was let go would be given out here, and written at once
            for size in (1 << 9, 1 << 14, 1 << 20, 10 << 20, 40 << 20):
                mine.append(torch.full((size,), 0x7f, dtype=torch.uint8, device=DEV))
        torch.cuda.current_stream().synchronize()
        assert all(bool((m == 0x7f).all()) for m in mine)
        torch.cuda.current_stream().wait_stream(other)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert all(bool((m == 0x7f).all()) for m in mine)
        del got, mine


def test_results_let_go_while_the_current_stream_reads_them(vl):
    X = operands(torch.bfloat16)[0]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    Q, E = vl.velora_checkpoint_store(X, stream=other)
    want = vl.velora_checkpoint_load(Q, E, stream=other)
    torch.cuda.synchronize()
    want = want.clone()
    zeros = torch.zeros_like(Q)
    torch.cuda.synchronize()
    got = vl.velora_checkpoint_load(Q, E, stream=other)
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda._sleep(20_000_000)
    copy = got + 0                                             # reads it some 10 ms from now
    del got
    for _ in range(4):
        vl.velora_checkpoint_load(zeros, E, stream=other)      # would write it at once
    torch.cuda.synchronize()
    assert torch.equal(copy, want)
