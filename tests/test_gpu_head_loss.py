"""Cross entropy of a linear head and its gradients on the GPU against the definition in 64 bits.

Bounds, element by element, from the arithmetic (u = 2^-24; sums of K products of bf16 numbers are exact products added by the tensor
cores with truncation, K / 16 times into the accumulator; of fp32 numbers K roundings):
  logits   d = (K / 16 + 16) 2u max_v sum |x w|  (bf16),   K 2u max_v sum |x w|  (fp32)
  loss     2 d from the two logits' errors (log sum exp moves by no more than its arguments), exp and log: 2^-19 + 4u |lse|
  G        g (p (2 d + 2^-18 + 4u |lse|)), and half a step of bf16, 2^-8 |G|, where it is stored so; 2^-16 |G| as two of them (up to 64 tokens)
  dX, dW   sum |error of G| |factor|, the products' sums like the logits', half a step of the output's type
"""
import numpy as np
import pytest
import torch

from _util import Guard

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


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


def batch(N, D, V, dtype, seed, masked="none", scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    W = (torch.randn((V, D), generator=g, device=DEV) / D ** 0.5).to(dtype)
    t = torch.randint(V, (N,), generator=g, device=DEV)
    X = ((torch.randn((N, D), generator=g, device=DEV) + 6 * torch.rand((N, 1), generator=g, device=DEV) * W[t].float()) * scale).to(dtype)
    if masked == "some":
        t = torch.where(torch.rand(N, generator=g, device=DEV) < 0.6, -100, t)
    elif masked == "all":
        t = torch.full_like(t, -1)
    elif masked == "all but the last":
        t[:-1] = -100
    elif masked == "every other":
        t[::2] = -2 ** 40
    dloss = torch.randn(N, generator=g, device=DEV)
    return X, W, t, dloss


def sums(K, dtype):
    return (K / 16 + 16) * 2 * U if dtype == torch.bfloat16 else K * 2 * U


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


class Reference:
    def __init__(self, X, W, target, dloss):
        dtype, V = X.dtype, W.shape[0]
        self.live = (target >= 0) & (target < V)
        x, w = torch.where(self.live[:, None], X.double(), 0.0), W.double()
        t = torch.where(self.live, target, 0)
        l = x @ w.t()
        lse = torch.logsumexp(l, 1)
        hit = l.gather(1, t[:, None])[:, 0]
        d = sums(X.shape[1], dtype) * (x.abs() @ w.abs().t()).amax(1)
        zero = torch.zeros_like(lse)
        self.loss, self.lse = torch.where(self.live, lse - hit, zero), torch.where(self.live, lse, zero)
        self.loss_bound = torch.where(self.live, 2 * d + 2.0 ** -19 + 4 * U * (lse.abs() + hit.abs()), zero)
        g = torch.where(self.live, dloss.double(), zero)
        p = torch.exp(l - lse[:, None])
        G = p * g[:, None]
        G.scatter_add_(1, t[:, None], -g[:, None])
        rounding = (half_step(dtype) if X.shape[0] > 64 else half_step(dtype) ** 2) if dtype == torch.bfloat16 else 4 * U
        dG = g.abs()[:, None] * p * (2 * d + 2.0 ** -18 + 4 * U * lse.abs())[:, None] + rounding * G.abs()
        self.dX, self.dW = G @ w, G.t() @ x
        self.dX_bound = dG @ w.abs() + sums(V, dtype) * (G.abs() @ w.abs())
        self.dW_bound = dG.t() @ x.abs() + sums(X.shape[0], dtype) * (G.abs().t() @ x.abs())


def check(got, ref, bound, what, out_rounding):
    bound = bound + (out_rounding + U) * ref.abs() + 1e-30
    diff = (got.double() - ref).abs()
    assert bool(torch.isfinite(got).all()), what
    worst = (diff / bound).max().item() if diff.numel() else 0.0
    assert worst <= 1.0, "%s: %.3g times its bound" % (what, worst)


def check_norm(got, ref, dtype, what, tokens):
    """Two independent roundings to bf16 (of G, of the output), each at most half a step: their norms add in squares.  One up to 64 tokens."""
    if dtype == torch.bfloat16 and ref.norm() > 0:
        assert (got.double() - ref).norm() <= (2 ** 0.5 if tokens > 64 else 1.01) * 2.0 ** -8 * ref.norm(), what


SIZES = [(1, 8, 1), (1, 64, 100), (2, 16, 33), (64, 768, 1000), (63, 128, 3000), (5, 1024, 3001), (200, 520, 2500), (3, 72, 257), (65, 128, 1000), (300, 256, 2049), (257, 512, 4097), (1030, 264, 777), (129, 1024, 8192)]


@pytest.mark.parametrize("masked", ["none", "some", "all", "all but the last", "every other"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V", SIZES)
def test_loss_and_gradients(vl, guard, N, D, V, dtype, masked):
    X, W, t, dloss = batch(N, D, V, dtype, N + D + V, masked)
    ref = Reference(X, W, t, dloss)
    f32 = vl.OP_F32 if dtype == torch.float32 else 0
    ws = guard.workspace(vl, vl.velora_workspace_bytes(vl.OP_HEAD_LOSS | f32, N, D, V, 1, False))
    loss, lse = vl.velora_head_loss(X, W, t, guard.vec(N), guard.vec(N), ws=ws)
    check(loss, ref.loss, ref.loss_bound, "loss", 0)
    check(lse, ref.lse, ref.loss_bound, "lse", 0)
    assert vl.velora_workspace_status(ws) == 0
    ws = guard.workspace(vl, vl.velora_workspace_bytes(vl.OP_HEAD_LOSS_BACKWARD | f32, N, D, V, 1, False))
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, dloss, guard.mat(N, D, dtype), guard.mat(V, D, dtype), ws=ws)
    check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
    check(dW, ref.dW, ref.dW_bound, "dW", half_step(dtype))
    check_norm(dX, ref.dX, dtype, "dX", N)
    check_norm(dW, ref.dW, dtype, "dW", N)
    assert bool((dX[~ref.live] == 0).all())
    assert vl.velora_workspace_status(ws) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V", [(70, 77, 501), (200, 136, 1031)])
def test_any_rows_and_accumulation(vl, guard, N, D, V, dtype):
    """Dense rows of an odd width, views that start anywhere, fp32 and bf16 dW with beta = 1, one gradient without the other."""
    X, W, t, dloss = batch(N, D, V, dtype, 5, "some")
    ref = Reference(X, W, t, dloss)

    def moved(x):
        buf = torch.full((x.shape[0], x.shape[1] + 5), float("nan"), device=DEV, dtype=x.dtype)
        buf[:, 3:3 + x.shape[1]] = x
        return buf[:, 3:3 + x.shape[1]]

    for x, w in ((X, W), (moved(X), W), (X, moved(W)), (moved(X), moved(W))):
        loss, lse = vl.velora_head_loss(x, w, t)
        check(loss, ref.loss, ref.loss_bound, "loss", 0)
        for dw_dtype in (torch.float32, torch.bfloat16):
            start = torch.randn((V, D), device=DEV).to(dw_dtype)
            dX, dW = guard.mat(N, D, dtype, ld=D + 1), guard.mat(V, D, dw_dtype, ld=D + 3, init=start)
            vl.velora_head_loss_backward(x, w, t, lse, dloss, dX, dW, beta=1)
            check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
            check(dW, ref.dW + start.double(), ref.dW_bound + 2 * U * start.double().abs(), "dW", half_step(dw_dtype))
        none, dW = vl.velora_head_loss_backward(x, w, t, lse, dloss, need_dX=False, dw_dtype=torch.float32)
        assert none is None
        check(dW, ref.dW, ref.dW_bound, "dW alone", 0)
        dX, none = vl.velora_head_loss_backward(x, w, t, lse, dloss, need_dW=False)
        assert none is None
        check(dX, ref.dX, ref.dX_bound, "dX alone", half_step(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_stands_in_tokens_without_a_target_does_not_matter(vl, dtype):
    N, D, V = 150, 200, 700
    X, W, t, dloss = batch(N, D, V, dtype, 8, "some")
    loss, lse = vl.velora_head_loss(X, W, t)
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, dloss)
    dead = t < 0
    Y, s, g = X.clone(), lse.clone(), dloss.clone()
    Y[dead] = float("nan")
    Y[dead.nonzero()[0, 0]] = float("inf")
    s[dead] = float("nan")
    g[dead] = float("inf")
    loss2, lse2 = vl.velora_head_loss(Y, W, t)
    dX2, dW2 = vl.velora_head_loss_backward(Y, W, t, s, g)
    for a, b in ((loss, loss2), (lse, lse2), (dX, dX2), (dW, dW2)):
        assert torch.equal(a, b)
    assert bool((loss[dead] == 0).all()) and bool((lse[dead] == 0).all()) and bool((dX[dead] == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_target_that_is_no_column(vl, dtype):
    N, D, V = 40, 64, 300
    X, W, t, dloss = batch(N, D, V, dtype, 12)
    t[7], t[39] = V, 2 ** 40
    ref = Reference(X, W, t, dloss)
    ws = vl.velora_workspace_alloc(vl.velora_workspace_bytes(vl.OP_HEAD_LOSS_BACKWARD | (vl.OP_F32 if dtype == torch.float32 else 0), N, D, V, 1), DEV)
    loss, lse = vl.velora_head_loss(X, W, t, ws=ws)
    bad = ~ref.live
    assert int(bad.sum()) == 2 and bool(torch.isnan(loss[bad]).all())
    check(loss[~bad], ref.loss[~bad], ref.loss_bound[~bad], "loss", 0)
    from paper_2405_17991_b200 import binding
    assert vl.velora_workspace_status(ws) == binding.ERR_INVALID_ARG
    vl.velora_workspace_init(ws)
    assert vl.velora_workspace_status(ws) == 0
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, dloss, ws=ws)
    assert vl.velora_workspace_status(ws) == binding.ERR_INVALID_ARG
    check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
    check(dW, ref.dW, ref.dW_bound, "dW", half_step(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [1e-3, 30.0])
def test_flat_and_steep_distributions(vl, dtype, scale):
    """Logits near zero, and up to hundreds: exponentials that vanish beside the largest."""
    N, D, V = 100, 128, 3001
    X, W, t, dloss = batch(N, D, V, dtype, 31, scale=scale)
    ref = Reference(X, W, t, dloss)
    loss, lse = vl.velora_head_loss(X, W, t)
    check(loss, ref.loss, ref.loss_bound, "loss", 0)
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, dloss)
    check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
    check(dW, ref.dW, ref.dW_bound, "dW", half_step(dtype))


def test_non_finite_rows_stay_with_their_token(vl):
    """A token with a target and a NaN: its loss is NaN, the others' are not."""
    N, D, V = 300, 64, 500
    X, W, t, dloss = batch(N, D, V, torch.bfloat16, 40)
    X[3, 5] = float("nan")
    loss, _ = vl.velora_head_loss(X, W, t)
    ok = torch.arange(N, device=DEV) != 3
    assert bool(torch.isnan(loss[3])) and bool(torch.isfinite(loss[ok]).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_small_workspaces_mean_smaller_pieces(vl, guard, dtype):
    N, D, V = 300, 136, 5000
    X, W, t, dloss = batch(N, D, V, dtype, 50, "some")
    ref = Reference(X, W, t, dloss)
    f32 = vl.OP_F32 if dtype == torch.float32 else 0
    _, lse = vl.velora_head_loss(X, W, t)
    full = vl.velora_workspace_bytes(vl.OP_HEAD_LOSS_BACKWARD | f32, N, D, V, 1, False)
    tiny = vl.velora_workspace_bytes(vl.OP_HEAD_LOSS_BACKWARD | f32, N, D, 256, 1, False)      # a vocabulary of one piece
    assert tiny < full
    for size in (tiny, tiny + 2 * 256 * N * 4, full, 2 * full):
        ws = guard.workspace(vl, size)
        dX, dW = vl.velora_head_loss_backward(X, W, t, lse, dloss, ws=ws)
        check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
        check(dW, ref.dW, ref.dW_bound, "dW", half_step(dtype))
    with pytest.raises(vl.VeloraError):
        vl.velora_head_loss_backward(X, W, t, lse, dloss, ws=torch.zeros(4096, dtype=torch.uint8, device=DEV))


def test_gradients_against_differences(vl):
    """Central differences of the loss along random directions, fp32, h = 1/64.  The third derivative of log sum exp along a direction
    whose logits move by at most r is below 2 r^3, so the difference is off by h^2 r^3 / 3 a token and by the loss's error over h."""
    N, D, V = 20, 32, 60
    X, W, t, _ = batch(N, D, V, torch.float32, 60)
    g = torch.full((N,), 1.0 / N, device=DEV)
    loss, lse = vl.velora_head_loss(X, W, t)
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, g)
    err = (Reference(X, W, t, g).loss_bound.max() * 1.5).item()
    gen = torch.Generator(device=DEV).manual_seed(1)
    h = 1.0 / 64
    for which in range(2):
        P = X if which == 0 else W
        for _ in range(3):
            dirn = torch.randn(P.shape, generator=gen, device=DEV)
            dirn = dirn / dirn.norm()

            def total(s):
                q = P + s * dirn
                return vl.velora_head_loss(q if which == 0 else X, W if which == 0 else q, t)[0].double().mean().item()

            r = 2 * ((dirn @ W.t()).abs().max() if which == 0 else (X @ dirn.t()).abs().max()).item()
            slope = ((dX if which == 0 else dW).double() * dirn.double()).sum().item()
            # rounding of P + s dirn: half a step of values below 8, times the gradient
            moved = 8 * 2.0 ** -24 * (dX if which == 0 else dW).double().abs().sum().item() / h
            assert abs((total(h) - total(-h)) / (2 * h) - slope) <= h * h * r ** 3 / 3 + err / h + moved


def test_empty_batch(vl):
    X, W = torch.empty((0, 64), device=DEV, dtype=torch.bfloat16), torch.randn((30, 64), device=DEV).to(torch.bfloat16)
    t, none = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    loss, lse = vl.velora_head_loss(X, W, t)
    assert loss.shape == (0,) and lse.shape == (0,)
    dW = torch.ones_like(W)
    vl.velora_head_loss_backward(X, W, t, lse, none, dW=dW, beta=1)
    assert bool((dW == 1).all())
    dX, _ = vl.velora_head_loss_backward(X, W, t, lse, none, dW=dW)
    assert dX.shape == (0, 64) and bool((dW == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured_replayed_and_on_another_stream(vl, dtype):
    N, D, V = 200, 128, 1500
    first, second = (batch(N, D, V, dtype, s, m) for s, m in ((70, "some"), (71, "none")))
    want = []
    for X, W, t, g in (first, second):
        loss, lse = vl.velora_head_loss(X, W, t)
        want.append((loss, *vl.velora_head_loss_backward(X, W, t, lse, g)))
    f32 = vl.OP_F32 if dtype == torch.float32 else 0
    ws = vl.velora_workspace_alloc(vl.velora_workspace_bytes(vl.OP_HEAD_LOSS_BACKWARD | f32, N, D, V, 1), DEV)
    ws1 = vl.velora_workspace_alloc(vl.velora_workspace_bytes(vl.OP_HEAD_LOSS | f32, N, D, V, 1), DEV)
    X, W, t, g = (x.clone() for x in first)
    loss, lse = vl.velora_head_loss(X, W, t, ws=ws1)
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, g, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vl.velora_head_loss(X, W, t, loss, lse, ws=ws1)
        vl.velora_head_loss_backward(X, W, t, lse, g, dX, dW, ws=ws)
    for case, ref in ((second, want[1]), (first, want[0])):        # the number of targets differs from the captured one
        for mine, new in zip((X, W, t, g), case):
            mine.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, ref[0]) and torch.equal(dX, ref[1]) and torch.equal(dW, ref[2])
    # two streams at once, a workspace each
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, (X, W, t, g) in zip(streams, (first, second)):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            loss, lse = vl.velora_head_loss(X, W, t)
            got.append((loss, *vl.velora_head_loss_backward(X, W, t, lse, g)))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("power", [10, 20, 24, 30, 60, 100])
@pytest.mark.parametrize("N", [3, 100, 200])
def test_logits_of_any_size(vl, N, power, dtype):
    """Logits 2^power (v - 50): each is exact, and the row's largest alone has a share in the sum, so loss and lse are exact as well.

    The share itself, 1, is one in fp32, exp(0).  In bf16 it is 2^y (1 - y ln 2) with y, what the rounding of lse log2 e loses, up to 2^-8: off by
    (y ln 2)^2 / 2 < 3.7e-6 and 2^-22 of the exponential, together below 2^-17."""
    V, D = 100, 64
    W = torch.randint(-7, 8, (V, D), device=DEV).to(dtype)
    W[:, 0] = torch.arange(V, device=DEV) - 50
    X = torch.zeros((N, D), device=DEV, dtype=dtype)
    sign = torch.where(torch.arange(N, device=DEV) % 3 == 0, -1.0, 1.0)
    X[:, 0] = sign * 2.0 ** power
    top = torch.where(sign > 0, V - 1, 0)
    t = torch.where(torch.arange(N, device=DEV) % 2 == 0, top, torch.randint(V, (N,), device=DEV))
    loss, lse = vl.velora_head_loss(X, W, t)
    logits = X.double() @ W.double().t()
    assert torch.equal(lse.double(), logits.amax(1))
    assert torch.equal(loss, lse - logits.gather(1, t[:, None])[:, 0].float())
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, torch.ones(N, device=DEV))
    share = 2.0 ** -17 if dtype == torch.bfloat16 else 0.0
    of_top, of_target = (torch.nn.functional.one_hot(c, V).double() for c in (top, t))
    ref, bound = (of_top - of_target) @ W.double(), share * of_top @ W.double().abs()
    assert bool(((dX.double() - ref).abs() <= (1 + share) * (bound + half_step(dtype) * ref.abs())).all())
    ref, bound = (of_top - of_target).t() @ X.double(), share * of_top.t() @ X.double().abs()
    assert bool(((dW.double() - ref).abs() <= (1 + share) * (bound + half_step(dtype) * ref.abs())).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,shift", [(100, 25), (150, 24)])
def test_rows_past_32_bits(vl, N, shift, dtype):
    """Pitches that put the last rows of X, W, dX and dW more than 2^31 elements behind the first."""
    D, V = 64, 600
    X, W, t, dloss = batch(N, D, V, dtype, 7, "some")
    ref = Reference(X, W, t, dloss)

    def far(rows, shift):
        assert (rows - 1) << shift > 2 ** 31
        return torch.empty_strided((rows, D), (1 << shift, 1), dtype=dtype, device=DEV)

    x, w, dX, dW = far(N, shift), far(V, 22), far(N, shift), far(V, 22)
    x.copy_(X)
    w.copy_(W)
    loss, lse = vl.velora_head_loss(x, w, t)
    check(loss, ref.loss, ref.loss_bound, "loss", 0)
    vl.velora_head_loss_backward(x, w, t, lse, dloss, dX, dW)
    check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
    check(dW, ref.dW, ref.dW_bound, "dW", half_step(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_more_than_2_to_31_logits_at_a_time(vl, dtype):
    N, D, V = 2200000, 16, 1500
    X, W, t, dloss = batch(N, D, V, dtype, 8, "some")
    loss, lse = vl.velora_head_loss(X, W, t)
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, dloss)
    want, bound = 0.0, 0.0
    for at in range(0, N, 1 << 17):
        part = slice(at, at + (1 << 17))
        ref = Reference(X[part], W, t[part], dloss[part])
        check(loss[part], ref.loss, ref.loss_bound, "loss", 0)
        check(dX[part], ref.dX, ref.dX_bound, "dX", half_step(dtype))
        want, bound = want + ref.dW, bound + ref.dW_bound * (sums(N, dtype) / sums(1 << 17, dtype))
    check(dW, want, bound, "dW", half_step(dtype))
