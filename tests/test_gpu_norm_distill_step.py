"""The pieces as a student's training step uses them: a residual stream normed in front of a VeLoRA layer whose output goes back to it, a final norm, a head
taught by a teacher; then backwards through all of it, over two micro-batches added up, eagerly and from a CUDA graph.

Every gradient is compared with the chain's in 64 bits from the same bf16 weights and inputs (v and Z's projection included).  Bound, norm-wise: each stored
bf16 tensor on the way (H0, Y0, A, H1, Y1, G, dY1, dH1, dA's product, dY0, the output) is off by at most half a step, 2^-8, of its own norm, and the factored
gradient's Z by another; twelve of them passed on by products that are no worse conditioned than sums of random signs, and by norms, which keep a row's scale:
sqrt(12) * 2^-8 = 1.35e-2, twice that as the bound.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
BOUND = 2 * 12 ** 0.5 * 2.0 ** -8
N, D, V, K, DSUB, T = 520, 512, 3001, 20, 64, 2.0


@pytest.fixture(scope="module")
def vl():
    import paper_2405_17991_b200 as pkg
    pkg.lib()
    return pkg


def problem():
    g = torch.Generator(device=DEV)
    g.manual_seed(21)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    weights = {"W": (r(D, D) / D ** 0.5).bfloat16(), "head": (r(V, D) / D ** 0.5).bfloat16(), "w0": 1 + 0.2 * r(D), "b0": 0.1 * r(D), "w1": 1 + 0.2 * r(D),
               "b1": 0.1 * r(D)}
    batches = []
    for _ in range(2):
        i = torch.randint(V, (N, K), generator=g, device=DEV)
        i = torch.where(torch.rand((N, 1), generator=g, device=DEV) < 0.3, -1, i)
        batches.append({"X": r(N, D).bfloat16(), "R": r(N, D).bfloat16(), "i": i, "t": 2 * r(N, K)})
    v = r(DSUB)
    return weights, v / v.norm(), batches


def norm64(h, w, b):
    c = h - h.mean(1, keepdim=True)
    s = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5)
    return c * s * w + b, c * s, s


def norm64_back(dy, xhat, s, w):
    c = dy * w
    return s * (c - c.mean(1, keepdim=True) - xhat * (c * xhat).mean(1, keepdim=True)), (dy * xhat).sum(0), dy.sum(0)


def reference(weights, v, batches):
    p = {k: x.double() for k, x in weights.items()}
    v = v.double()
    total = {k: torch.zeros_like(x) for k, x in p.items()}
    loss, dXs = 0.0, []
    for q in batches:
        h0 = q["X"].double() + q["R"].double()
        y0, x0, s0 = norm64(h0, p["w0"], p["b0"])
        z = y0.view(N, -1, DSUB) @ v
        y0hat = (z[:, :, None] * v).reshape(N, D)
        h1 = h0 + y0 @ p["W"].t()
        y1, x1, s1 = norm64(h1, p["w1"], p["b1"])
        l = y1 @ p["head"].t() / T
        lse = torch.logsumexp(l, 1)
        some = q["i"] >= 0
        live = some.any(1)
        u = torch.where(some, q["t"].double() / T, -float("inf"))
        prob = torch.where(live[:, None], torch.softmax(torch.where(live[:, None], u, 0.0), 1), 0.0)
        col = q["i"].clamp(min=0)
        g = live.double() / live.sum()
        loss += (g[:, None] * prob * (torch.log(prob.clamp(min=1e-300)) - l.gather(1, col) + lse[:, None])).sum()
        G = torch.exp(l - lse[:, None])
        G = (g / T)[:, None] * (G * prob.sum(1, keepdim=True)).scatter_add(1, col, -prob)
        total["head"] += G.t() @ y1
        dh1, dw, db = norm64_back(G @ p["head"], x1, s1, p["w1"])
        total["w1"] += dw
        total["b1"] += db
        total["W"] += dh1.t() @ y0hat
        dy0 = dh1 @ p["W"]
        dh0, dw, db = norm64_back(dy0, x0, s0, p["w0"])
        total["w0"] += dw
        total["b0"] += db
        dXs.append(dh0 + dh1)
    return loss, total, dXs


class Step:
    def __init__(self, vl, weights, v, batches):
        self.vl, self.p, self.v, self.batches = vl, weights, v, batches
        size = vl.velora_workspace_bytes
        need = max(size(vl.OP_LINEAR_FORWARD, N, D, D, DSUB), size(vl.OP_LINEAR_BACKWARD_FACTORED, N, D, D, DSUB), size(vl.OP_HEAD_DISTILL, N, D, V, K),
                   size(vl.OP_HEAD_DISTILL_BACKWARD, N, D, V, K), size(vl.OP_LAYER_NORM_BACKWARD, N, D, 1, 1))
        self.ws = vl.velora_workspace_alloc(need, DEV)             # one workspace for everything, calls in one stream
        self.grads = {k: torch.zeros(w.shape, device=DEV) for k, w in weights.items()}
        self.losses = [torch.empty(N, device=DEV) for _ in batches]
        self.dXs = [torch.empty_like(q["X"]) for q in batches]
        self.dloss = [((q["i"] >= 0).any(1).float() / (q["i"] >= 0).any(1).sum()).contiguous() for q in batches]

    def run(self):
        vl, ws, p, g = self.vl, self.ws, self.p, self.grads
        for n, q in enumerate(self.batches):
            beta = 1 if n else 0
            Y0, H0, m0, r0 = vl.velora_layer_norm(q["X"], p["w0"], p["b0"], residual=q["R"])
            A, Z = vl.velora_linear_forward(Y0, p["W"], self.v, ws=ws)
            Y1, H1, m1, r1 = vl.velora_layer_norm(A, p["w1"], p["b1"], residual=H0, Y=A)       # A is not needed any more
            _, lse = vl.velora_head_distill(Y1, p["head"], q["i"], q["t"], T, loss=self.losses[n], ws=ws)
            dY1, _ = vl.velora_head_distill_backward(Y1, p["head"], q["i"], q["t"], lse, self.dloss[n], T, dW=g["head"], beta=beta, ws=ws)
            dH1, _, _ = vl.velora_layer_norm_backward(dY1, H1, m1, r1, p["w1"], dweight=g["w1"], dbias=g["b1"], beta=beta, ws=ws)
            dY0, _ = vl.velora_linear_backward(dH1, p["W"], Z, self.v, dW=g["W"], beta=beta, ws=ws)
            vl.velora_layer_norm_backward(dY0, H0, m0, r0, p["w0"], dH=dH1, dX=self.dXs[n], dweight=g["w0"], dbias=g["b0"], beta=beta, ws=ws)


def test_step_of_two_micro_batches(vl):
    parts = problem()
    loss, total, dXs = reference(*parts)
    step = Step(vl, *parts)
    step.run()
    got = sum((x.double() * g.double()).sum() for x, g in zip(step.losses, step.dloss))
    assert abs(got - loss) <= BOUND * abs(loss)
    results = {**{k: (step.grads[k], total[k]) for k in total}, **{"dX%d" % i: (step.dXs[i], dXs[i]) for i in range(2)}}
    for name, (x, ref) in results.items():
        assert (x.double() - ref).norm() <= BOUND * ref.norm(), name
    assert vl.velora_workspace_status(step.ws) == 0
    eager = [x.clone() for x, _ in results.values()]
    # the same bits from a graph, twice, and from the same calls again
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    outs = [x for x, _ in results.values()]
    for _ in range(2):
        for x in outs:
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
    step.run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, eager))
    # and through the current stream of a thread's own, two steps at once, a workspace each
    other = Step(vl, *parts)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s, one in zip(streams, (step, other)):
        with torch.cuda.stream(s):
            one.run()
    torch.cuda.synchronize()
    for one in (step, other):
        assert all(torch.equal(a, b) for a, b in zip([one.grads[k] for k in total] + one.dXs, eager))
