"""Gradients of tokens that the head is already sure of: there G[n, t] = g (exp(l - lse) - 1) cancels, and whatever the two passes' logits differ
by comes out divided by 1 - p.

Bounds, element by element, u = 2^-24, p the shares, d the error of a logit (test_gpu_head_loss):
  both passes add a logit up in the same way, so its error moves p_t and lse together: dp_t = p_t (1 - p_t) 2 d, dp_v = p_v 2 d for the others;
  lse is rounded to fp32 and its sum of exponentials, near one where a token is sure, by u at each of at most 2^6 additions on a column's way
  through segments of 128 columns, slices and blocks; exponential and products 2^-22 each: together p (2^-18 + 4 u |lse|);
  G's own rounding, the products' sums and the output's as in test_gpu_head_loss.
An fp32 product's form goes by its size, so a slice's logits may be added up in another order than the whole batch's.  Each order is off by at
most d, so shares differ by up to p 2 d there.
A row is compared by its norm with the norm of its elements' bounds."""
import pytest
import torch

from test_gpu_head_loss import U, half_step, sums

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def vl():
    import paper_2405_17991_b200 as pkg
    pkg.lib()
    return pkg


def sure_batch(N, D, V, dtype, negative, seed):
    """Target logits 12 to 19 above the others' typical one; `negative`: with a direction that all columns share and that takes 28 off every logit."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    W = r(V, D) / D ** 0.5
    shared = r(D)
    shared = shared / shared.norm()
    if negative:
        W = W + 0.5 * shared
    t = torch.randint(V, (N,), generator=g, device=DEV)
    own = W[t] - (0.5 * shared if negative else 0.0)
    X = r(N, D) + (12 + 7 * torch.rand((N, 1), generator=g, device=DEV)) * own
    if negative:
        X = X - 56 * shared
    return X.to(dtype), W.to(dtype), t, torch.rand(N, generator=g, device=DEV) + 0.5


class SureReference:
    def __init__(self, X, W, t, dloss, tokens, same_sums=True):
        dtype, V = X.dtype, W.shape[0]
        x, w, g = X.double(), W.double(), dloss.double()
        l = x @ w.t()
        lse = torch.logsumexp(l, 1)
        p = torch.exp(l - lse[:, None])
        self.loss, self.hit = lse - l.gather(1, t[:, None])[:, 0], l.gather(1, t[:, None])[:, 0]
        d = sums(X.shape[1], dtype) * (x.abs() @ w.abs().t()).amax(1)
        G = p * g[:, None]
        G.scatter_add_(1, t[:, None], -g[:, None])
        moved = p * 2 * d[:, None]
        at = p.gather(1, t[:, None])
        if same_sums:
            moved.scatter_(1, t[:, None], at * -torch.expm1(-self.loss)[:, None] * 2 * d[:, None])
        rounding = (half_step(dtype) if tokens > 64 else half_step(dtype) ** 2) if dtype == torch.bfloat16 else 4 * U
        dG = g[:, None] * (moved + p * (2.0 ** -18 + 4 * U * lse.abs())[:, None]) + rounding * G.abs()
        self.dX, self.dW = G @ w, G.t() @ x
        self.dX_bound = dG @ w.abs() + sums(V, dtype) * (G.abs() @ w.abs()) + half_step(dtype) * self.dX.abs()
        self.dW_bound = dG.t() @ x.abs() + sums(X.shape[0], dtype) * (G.abs().t() @ x.abs()) + half_step(dtype) * self.dW.abs()


def check_rows(got, ref, bound, what):
    worst = ((got.double() - ref).norm(dim=1) / bound.norm(dim=1).clamp(min=1e-30)).max().item()
    assert worst <= 1.0, "%s: a row off by %.3g times its bound" % (what, worst)


@pytest.mark.parametrize("negative", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [2048, 4096])
@pytest.mark.parametrize("N", [1, 8, 64, 100, 300])
def test_gradients_of_sure_tokens(vl, N, D, dtype, negative):
    V = 2000
    X, W, t, dloss = sure_batch(N, D, V, dtype, negative, N + D)
    ref = SureReference(X, W, t, dloss, N)
    if N >= 64:
        assert ref.loss.median() < 5e-3 and bool((ref.hit < 0).all() if negative else (ref.hit > 0).all())
    loss, lse = vl.velora_head_loss(X, W, t)
    dX, dW = vl.velora_head_loss_backward(X, W, t, lse, dloss)
    check_rows(dX, ref.dX, ref.dX_bound, "dX")
    hit = torch.unique(t)                                      # columns of other tokens alone have rows too small to tell
    check_rows(dW[hit], ref.dW[hit], ref.dW_bound[hit], "dW")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("step", [40, 100, 150])
def test_backward_pass_of_a_slice_of_the_tokens(vl, step, dtype):
    """lse of the whole batch, gradients a slice at a time: another kernel has to form the same logits."""
    N, D, V = 300, 4096, 2000
    X, W, t, dloss = sure_batch(N, D, V, dtype, False, 5)
    _, lse = vl.velora_head_loss(X, W, t)
    for at in range(0, N, step):
        s = slice(at, at + step)
        n = X[s].shape[0]
        ref = SureReference(X[s], W, t[s], dloss[s], n, dtype == torch.bfloat16)
        dX, _ = vl.velora_head_loss_backward(X[s], W, t[s], lse[s].contiguous(), dloss[s].contiguous(), need_dW=False)
        check_rows(dX, ref.dX, ref.dX_bound, "dX")


@pytest.mark.parametrize("D", [64, 500, 576, 4096])
def test_every_kernel_forms_the_same_logits(vl, D):
    """With one column lse is the logit itself, so its bits are to be seen: the kernel for more than 128 tokens, those for up to 128, 64 and 32."""
    g = torch.Generator(device=DEV)
    g.manual_seed(D)
    N = 1200
    X, W = torch.randn((N, D), generator=g, device=DEV).bfloat16(), torch.randn((1, D), generator=g, device=DEV).bfloat16()
    t = torch.zeros(N, dtype=torch.int64, device=DEV)
    whole = vl.velora_head_loss(X, W, t)[1]
    for step in (200, 100, 60, 30, 1):
        assert torch.equal(torch.cat([vl.velora_head_loss(X[i:i + step], W, t[i:i + step])[1] for i in range(0, N, step)]), whole)
