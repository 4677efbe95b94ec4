"""A training step as the pieces are used together: a layer whose input is kept in 8 bits, a VeLoRA layer, a linear head with its loss; two
micro-batches added up, eagerly and from a CUDA graph.

Every gradient is compared with the chain's in 64 bits from the same bf16 weights and inputs (Xhat, v and Z's projection included).
Bound, norm-wise: each stored bf16 tensor on the way (Y1, Y2, G, dY2, dY1, the output) is off by at most half a step, 2^-8, of its own norm, the
factored gradient's Z by another; seven of them passed on by products that are no worse conditioned than sums of random signs: sqrt(7) * 2^-8 =
1.04e-2, twice that as the bound.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
BOUND = 2 * 7 ** 0.5 * 2.0 ** -8
N, D, H, O, V, DSUB = 520, 512, 1032, 768, 3001, 64


@pytest.fixture(scope="module")
def vl():
    import paper_2405_17991_b200 as pkg
    pkg.lib()
    return pkg


def problem():
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    W1, W2, W3 = (r(H, D) / D ** 0.5).bfloat16(), (r(O, H) / H ** 0.5).bfloat16(), (r(V, O) / O ** 0.5).bfloat16()
    batches = []
    for _ in range(2):
        X = (r(N, D) * torch.exp(0.5 * r(D))).bfloat16()
        t = torch.randint(V, (N,), generator=g, device=DEV)
        t = torch.where(torch.rand(N, generator=g, device=DEV) < 0.4, -100, t)
        batches.append((X, t))
    v = r(DSUB)
    return W1, W2, W3, v / v.norm(), batches


def reference(W1, W2, W3, v, batches):
    w1, w2, w3 = W1.double(), W2.double(), W3.double()
    total = {k: 0.0 for k in ("loss", "dW1", "dW2", "dW3")}
    for X, t in batches:
        from test_gpu_checkpoint import definition
        x = X.double()
        xhat = torch.from_numpy(definition(X)[2]).to(DEV)
        y1 = x @ w1.t()
        y2 = y1 @ w2.t()
        l = y2 @ w3.t()
        live = t >= 0
        g = live.double() / live.sum()
        lse = torch.logsumexp(l, 1)
        tt = t.clamp(min=0)
        total["loss"] += (g * (lse - l.gather(1, tt[:, None])[:, 0])).sum()
        G = torch.exp(l - lse[:, None]) * g[:, None]
        G.scatter_add_(1, tt[:, None], -g[:, None])
        dy2 = G @ w3
        dy1 = dy2 @ w2
        m = -(-H // DSUB)
        pad = torch.zeros((N, m * DSUB), dtype=torch.float64, device=DEV)
        pad[:, :H] = y1
        y1hat = ((pad.view(N, m, DSUB) @ v.double())[:, :, None] * v.double()).reshape(N, -1)[:, :H]
        total["dW3"] += G.t() @ y2
        total["dW2"] += dy2.t() @ y1hat
        total["dW1"] += dy1.t() @ xhat
    return total


class Step:
    def __init__(self, vl, W1, W2, W3, v, batches):
        self.vl, self.W1, self.W2, self.W3, self.v, self.batches = vl, W1, W2, W3, v, batches
        size = vl.velora_workspace_bytes
        need = max(size(vl.OP_LINEAR_FORWARD, N, H, O, DSUB), size(vl.OP_LINEAR_BACKWARD_FACTORED, N, H, O, DSUB), size(vl.OP_CHECKPOINT_WEIGHT_GRAD, N, D, H, 1),
                   size(vl.OP_HEAD_LOSS, N, O, V, 1), size(vl.OP_HEAD_LOSS_BACKWARD, N, O, V, 1))
        self.ws = vl.velora_workspace_alloc(need, DEV)             # one workspace for everything, calls in one stream
        self.dW1, self.dW2, self.dW3 = (torch.zeros(w.shape, device=DEV) for w in (W1, W2, W3))
        self.losses = [torch.empty(N, device=DEV) for _ in batches]
        self.dloss = [((t >= 0).float() / (t >= 0).sum()).contiguous() for _, t in batches]

    def run(self):
        vl, ws = self.vl, self.ws
        for i, (X, t) in enumerate(self.batches):
            beta = 1 if i else 0
            Q, E = vl.velora_checkpoint_store(X)
            Y1 = vl.velora_dense_product(vl.PRODUCT_A_BT, X, self.W1, ws=ws)
            Y2, Z = vl.velora_linear_forward(Y1, self.W2, self.v, ws=ws)
            _, lse = vl.velora_head_loss(Y2, self.W3, t, loss=self.losses[i], ws=ws)
            dY2, _ = vl.velora_head_loss_backward(Y2, self.W3, t, lse, self.dloss[i], dW=self.dW3, beta=beta, ws=ws)
            dY1, _ = vl.velora_linear_backward(dY2, self.W2, Z, self.v, dW=self.dW2, beta=beta, ws=ws)
            vl.velora_checkpoint_weight_grad(dY1, Q, E, dW=self.dW1, beta=beta, ws=ws)


def test_step_of_two_micro_batches(vl):
    parts = problem()
    ref = reference(*parts)
    step = Step(vl, *parts)
    step.run()
    loss = sum((l.double() * g.double()).sum() for l, g in zip(step.losses, step.dloss))
    assert abs(loss - ref["loss"]) <= BOUND * abs(ref["loss"])
    eager = []
    for name in ("dW1", "dW2", "dW3"):
        got = getattr(step, name)
        assert (got.double() - ref[name]).norm() <= BOUND * ref[name].norm(), name
        eager.append(got.clone())
    assert vl.velora_workspace_status(step.ws) == 0
    # the same bits from a graph, twice, and from the same calls again
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for _ in range(2):
        for w in (step.dW1, step.dW2, step.dW3):
            w.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((step.dW1, step.dW2, step.dW3), eager))
    step.run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((step.dW1, step.dW2, step.dW3), eager))
