"""Distillation into a linear head from a teacher's top logits, and its gradients, on the GPU against the definition in 64 bits.

Bounds, element by element, from the arithmetic (u = 2^-24; see test_gpu_head_loss.py for the products' sums):
  logits   d = ((K / 16 + 16) 2u max_v sum |x w| (bf16), K 2u max_v sum |x w| (fp32), and 3u max |x w|-sum for the temperature) / T
  p        relative: t / T rounds twice, its difference to the largest or the given sum once, exp by 2 of its last places, the sum of K <= 1024 of
           them in branches of at most 40 additions:  rho = 6u (max |t / T| + |s|) + 64u
  loss     sum p (2 d + rho |log p - l + lse + 1| + 2^-20 + 4u (|l| + |lse| + |log p|)) + 40u sum |p (log p - l + lse)|
  G        |g| / T (q P (2 d + 2^-18 + 4u |lse| + rho) + p (rho + 4u)), and half a step of bf16, 2^-8 |G|, where it is stored so; 2^-16 |G| as two of
           them (up to 64 tokens); q the student's share, P the sum of p
  dX, dW   sum |error of G| |factor|, the products' sums like the logits', half a step of the output's type
"""
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


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def sums(K, dtype):
    return (K / 16 + 16) * 2 * U if dtype == torch.bfloat16 else K * 2 * U


def batch(N, D, V, K, dtype, seed, T=1.0, masked="none", whole=False, t_dtype=torch.float32):
    """Columns at random, some of them twice, a third of the entries missing here and there; a student that agrees with its teacher in part."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    W = (r(V, D) / D ** 0.5).to(dtype)
    i = torch.randint(V, (N, K), generator=g, device=DEV)
    X = (r(N, D) + 4 * torch.rand((N, 1), generator=g, device=DEV) * W[i[:, 0]].float()).to(dtype)
    t = (3 * r(N, K) + 5).to(t_dtype)
    i = torch.where(torch.rand((N, K), generator=g, device=DEV) < 0.3, -1 - i, i)
    if K > 2:
        i[:, 1] = i[:, 2]
    if masked == "some":
        i[torch.rand(N, generator=g, device=DEV) < 0.6] = -100
    elif masked == "all":
        i[:] = -1
    elif masked == "all but the last":
        i[:-1] = -100
        i[-1, 0] = V - 1
    elif masked == "minus infinity":                              # as good as missing: one entry, or all, of a token
        t[::2, 0] = -float("inf")
        t[::3] = -float("inf")
    lse = None
    if whole:
        u = torch.where(i >= 0, t.double() / T, -float("inf"))
        lse = (torch.logsumexp(u, 1) + 0.5 * torch.rand(N, generator=g, device=DEV)).float()
        lse = torch.where(torch.isfinite(lse), lse, 0.0)
    return {"X": X, "W": W, "i": i, "t": t, "lse": lse, "g": r(N), "T": T}


class Reference:
    def __init__(self, p):
        X, W, i, t, T = p["X"], p["W"], p["i"], p["t"].double(), p["T"]
        dtype, (N, D), V = X.dtype, X.shape, W.shape[0]
        bad = (i >= V).any(1)
        is_entry = (i >= 0) & (i < V)
        u = torch.where(is_entry, t / T, -float("inf"))
        self.live = (u != -float("inf")).any(1) & ~bad
        u = torch.where(self.live[:, None], u, 0.0)
        s = torch.logsumexp(u, 1) if p["lse"] is None else p["lse"].double()
        prob = torch.where(self.live[:, None] & is_entry, torch.exp(u - s[:, None]), 0.0)
        logp = torch.where(prob > 0, u - s[:, None], 0.0)
        x, w = torch.where(self.live[:, None], X.double(), 0.0), W.double()
        l = x @ w.t() / T
        lse = torch.logsumexp(l, 1)
        col = torch.where(is_entry, i, 0)
        hit = l.gather(1, col)
        size = (x.abs() @ w.abs().t()).amax(1)
        d = (sums(D, dtype) + 3 * U) * size / T
        finite = torch.where(torch.isfinite(u), u.abs(), 0.0).amax(1)
        rho = 6 * U * (finite + torch.where(torch.isfinite(s), s.abs(), 0.0)) + 64 * U
        terms = prob * (logp - hit + lse[:, None])
        zero = torch.zeros_like(lse)
        P = prob.sum(1)
        self.loss, self.lse = torch.where(self.live, terms.sum(1), zero), torch.where(self.live, lse, zero)
        each = 2 * d[:, None] + rho[:, None] * (logp - hit + lse[:, None] + 1).abs() + 2.0 ** -20 + 4 * U * (hit.abs() + lse[:, None].abs() + logp.abs())
        self.loss_bound = torch.where(self.live, (prob * each).sum(1) + 40 * U * terms.abs().sum(1), zero)
        self.lse_bound = torch.where(self.live, d + 2.0 ** -20 + 4 * U * lse.abs(), zero)
        g = torch.where(self.live, p["g"].double(), zero) / T
        q = torch.exp(l - lse[:, None]) * P[:, None]
        at = torch.zeros_like(q).scatter_add_(1, col, prob)
        G = g[:, None] * (q - at)
        rounding = (half_step(dtype) if N > 64 else half_step(dtype) ** 2) if dtype == torch.bfloat16 else 4 * U
        dG = g.abs()[:, None] * (q * (2 * d + 2.0 ** -18 + 4 * U * lse.abs() + rho)[:, None] + at * (rho + 4 * U)[:, None]) + rounding * G.abs()
        self.dX, self.dW = G @ w, G.t() @ x
        self.dX_bound = dG @ w.abs() + sums(V, dtype) * (G.abs() @ w.abs())
        self.dW_bound = dG.t() @ x.abs() + sums(N, dtype) * (G.abs().t() @ x.abs())


def check(got, ref, bound, what, rounding=0.0):
    bound = bound + (rounding + U) * ref.abs() + 1e-30
    diff = (got.double() - ref).abs()
    assert bool(torch.isfinite(got).all()), what
    worst = (diff / bound).max().item() if diff.numel() else 0.0
    assert worst <= 1.0, "%s: %.3g times its bound" % (what, worst)


def check_norm(got, ref, dtype, what, tokens):
    """Two independent roundings to bf16 (of G, of the output), each at most half a step: their norms add in squares.  One up to 64 tokens."""
    if dtype == torch.bfloat16 and ref.norm() > 0:
        assert (got.double() - ref).norm() <= (2 ** 0.5 if tokens > 64 else 1.01) * 2.0 ** -8 * ref.norm(), what


def forward(vl, p, **k):
    return vl.velora_head_distill(p["X"], p["W"], p["i"], p["t"], p["T"], p["lse"], **k)


def backward(vl, p, lse, **k):
    return vl.velora_head_distill_backward(p["X"], p["W"], p["i"], p["t"], lse, p["g"], p["T"], p["lse"], **k)


def f32(vl, dtype):
    return vl.OP_F32 if dtype == torch.float32 else 0


def run(vl, guard, p, dw_dtype=None):
    X, W = p["X"], p["W"]
    (N, D), V, K, dtype = X.shape, W.shape[0], p["i"].shape[1], X.dtype
    ref = Reference(p)
    odd = D % 8 != 0
    ws = guard.workspace(vl, vl.velora_workspace_bytes(vl.OP_HEAD_DISTILL | f32(vl, dtype), N, D, V, K, odd))
    loss, lse = forward(vl, p, loss=guard.vec(N), lse=guard.vec(N), ws=ws)
    check(lse, ref.lse, ref.lse_bound, "lse")
    check(loss, ref.loss, ref.loss_bound, "loss")
    assert vl.velora_workspace_status(ws) == 0
    ws = guard.workspace(vl, vl.velora_workspace_bytes(vl.OP_HEAD_DISTILL_BACKWARD | f32(vl, dtype), N, D, V, K, odd))
    dX, dW = backward(vl, p, lse, dX=guard.mat(N, D, dtype), dW=guard.mat(V, D, dw_dtype or dtype), ws=ws)
    check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
    check(dW, ref.dW, ref.dW_bound, "dW", half_step(dw_dtype or dtype))
    check_norm(dX, ref.dX, dtype, "dX", N)
    if dw_dtype is None:
        check_norm(dW, ref.dW, dtype, "dW", N)
    assert bool((dX[~ref.live] == 0).all()) and bool((loss[~ref.live] == 0).all())
    assert vl.velora_workspace_status(ws) == 0
    return ref


SIZES = [(1, 8, 1, 1), (1, 64, 100, 7), (2, 16, 33, 40), (64, 768, 1000, 10), (63, 128, 3000, 33), (5, 1024, 3001, 64), (200, 520, 2500, 3), (3, 72, 257, 100),
         (65, 128, 1000, 200), (300, 256, 2049, 64), (257, 512, 4097, 31), (1030, 264, 777, 12), (129, 1024, 8192, 128)]


@pytest.mark.parametrize("masked", ["none", "some", "all", "all but the last", "minus infinity"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V,K", SIZES)
def test_loss_and_gradients(vl, guard, N, D, V, K, dtype, masked):
    T, whole = ((1.0, False), (2.0, True), (1.5, False), (0.7, True))[(N + K) % 4]
    run(vl, guard, batch(N, D, V, K, dtype, N + D + V, T, masked, whole, torch.bfloat16 if N % 2 else torch.float32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V,K", [(20, 64, 5000, 1024), (150, 64, 5000, 1000), (300, 128, 700, 513), (90, 128, 130, 1024), (130, 64, 128, 64), (40, 80, 129, 2)])
def test_long_lists_and_small_vocabularies(vl, guard, N, D, V, K, dtype):
    """Up to the longest list; more entries than columns, so that most columns come several times; vocabularies around a block of 128 columns."""
    run(vl, guard, batch(N, D, V, K, dtype, 17, 1.0, "none", True))


@pytest.mark.parametrize("N", [1, 4, 5, 8, 9, 15, 16, 17])
@pytest.mark.parametrize("D,V", [(4, 3), (200, 1000), (203, 1001), (1664, 515), (2052, 700), (4099, 130), (9000, 260)])
def test_few_tokens_in_fp32(vl, guard, N, D, V):
    """Up to 16 tokens have products of their own: tokens on both sides of their sizes, rows that shared memory holds and longer ones, of any width."""
    run(vl, guard, batch(N, D, V, 3, torch.float32, N + D, 1.0, "some" if N > 4 else "none", True))
    p = batch(N, D, V, 3, torch.float32, 5)
    _, lse = forward(vl, p)
    ref = Reference(p)
    tiny = vl.velora_workspace_bytes(vl.OP_HEAD_DISTILL_BACKWARD | vl.OP_F32, N, D, 256, 3, False)         # fewer slices of dX's sums, and pieces of the vocabulary
    tiny -= (vl.velora_workspace_bytes(vl.OP_HEAD_DISTILL_BACKWARD | vl.OP_F32, N, D, 256, 3, False) - 256) // 2 if V <= 256 else -2 * N * (V // 128 + 2) - 256
    full = vl.velora_workspace_bytes(vl.OP_HEAD_DISTILL_BACKWARD | vl.OP_F32, N, D, V, 3, False)
    for size in (tiny, full):
        try:
            dX, dW = backward(vl, p, lse, ws=guard.workspace(vl, size))
        except vl.VeloraError:
            assert size == tiny and V <= 256                  # half of it may be too little
            continue
        check(dX, ref.dX, ref.dX_bound, "dX")
        check(dW, ref.dW, ref.dW_bound, "dW")


@pytest.mark.parametrize("dw_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N", [1, 7, 16])
@pytest.mark.parametrize("D,V,ld,offset", [(96, 300, 96, 0), (96, 300, 104, 8), (96, 300, 97, 0), (96, 300, 104, 3), (131, 4001, 131, 1), (513, 700, 516, 0), (1024, 9500, 1024, 0)])
def test_weight_gradient_of_few_tokens_anywhere(vl, N, D, V, ld, offset, dw_dtype):
    """dW in fp32 products' own kernel: rows on any boundary, added to or not, and nothing beside them touched."""
    p = batch(N, D, V, 4, torch.float32, N + D, 1.5)
    _, lse = forward(vl, p)
    ref = Reference(p)
    room = torch.randn(offset + V * ld + 64, device=DEV).to(dw_dtype)
    before = room.clone()
    for beta in (0, 1):
        dW = room[offset:offset + V * ld].as_strided((V, D), (ld, 1))
        old = dW.double() if beta else torch.zeros((V, D), dtype=torch.float64, device=DEV)
        backward(vl, p, lse, dW=dW, beta=beta, need_dX=False)
        # the sum's own bound, its rounding, and, with beta, one more of fp32
        check(dW, ref.dW + old, ref.dW_bound + 2.0 ** -23 * old.abs(), "dW", half_step(dw_dtype))
    inside = torch.zeros_like(room, dtype=torch.bool)
    inside[offset:offset + V * ld].as_strided((V, D), (ld, 1)).fill_(True)
    assert torch.equal(room[~inside], before[~inside])


def test_a_vocabulary_of_millions(vl, guard):
    """Columns and places in a list of 1024 that do not fit 32 bits together, and, at 1000 entries fewer, do."""
    for K in (1024, 24):
        run(vl, guard, batch(3, 8, 4200001, K, torch.bfloat16, 41, 1.0, "none", False))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [3, 64, 100, 300])
def test_where_entries_lie(vl, guard, N, dtype):
    """All entries in neighbouring columns, at every border of 16, 112, 128 and 256 columns, in the first and the last column, one column only."""
    D, V, K = 64, 1001, 40
    p = batch(N, D, V, K, dtype, 21)
    n = torch.arange(N, device=DEV)[:, None]
    k = torch.arange(K, device=DEV)[None, :]
    borders = torch.tensor([0, 1, 15, 16, 31, 32, 63, 64, 95, 96, 111, 112, 113, 127, 128, 129, 223, 224, 239, 240, 255, 256, 257, 383, 384, 511, 512, 767,
                            768, 895, 896, 959, 960, 991, 992, 998, 999, 1000, 0, 1000], device=DEV)
    for i in ((n * 13 + k) % V, borders[(k + n) % K], torch.where(k < 20, 0, V - 1).expand(N, K), (n % V).expand(N, K)):
        p["i"] = i.contiguous()
        run(vl, guard, p)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V", [(70, 77, 501), (200, 136, 1031), (9, 40, 300)])
def test_any_rows_and_accumulation(vl, guard, N, D, V, dtype):
    """Dense rows of an odd width, views that start anywhere, lists with pitches, fp32 and bf16 dW with beta = 1, one gradient without the other."""
    K = 9
    p = batch(N, D, V, K, dtype, 5, 2.0, "some", True, torch.bfloat16)
    ref = Reference(p)

    def moved(x, none):
        buf = torch.full((x.shape[0], x.shape[1] + 5), none, device=DEV, dtype=x.dtype)
        buf[:, 3:3 + x.shape[1]] = x
        return buf[:, 3:3 + x.shape[1]]

    lists = {**p, "i": moved(p["i"], 2 ** 40), "t": moved(p["t"], float("nan"))}
    for q in (p, lists, {**lists, "X": moved(p["X"], float("nan"))}, {**p, "W": moved(p["W"], float("nan"))}):
        loss, lse = forward(vl, q)
        check(loss, ref.loss, ref.loss_bound, "loss")
        for dw_dtype in (torch.float32, torch.bfloat16):
            start = torch.randn((V, D), device=DEV).to(dw_dtype)
            dX, dW = guard.mat(N, D, dtype, ld=D + 1), guard.mat(V, D, dw_dtype, ld=D + 3, init=start)
            backward(vl, q, lse, dX=dX, dW=dW, beta=1)
            check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
            check(dW, ref.dW + start.double(), ref.dW_bound + 2 * U * start.double().abs(), "dW", half_step(dw_dtype))
        none, dW = backward(vl, q, lse, need_dX=False, dw_dtype=torch.float32)
        assert none is None
        check(dW, ref.dW, ref.dW_bound, "dW alone")
        dX, none = backward(vl, q, lse, need_dW=False)
        assert none is None
        check(dX, ref.dX, ref.dX_bound, "dX alone", half_step(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [5, 150])
def test_what_stands_in_tokens_without_entries_does_not_matter(vl, dtype, N):
    p = batch(N, 200, 700, 12, dtype, 8, 1.0, "some", True)
    p["i"][0], p["i"][1, 0] = -1, 3
    loss, lse = forward(vl, p)
    dX, dW = backward(vl, p, lse)
    dead = (p["i"] < 0).all(1)
    q = {k: v.clone() if torch.is_tensor(v) else v for k, v in p.items()}
    s = lse.clone()
    q["X"][dead], q["t"][dead], q["g"][dead], q["lse"][dead], s[dead] = (float("nan"),) * 5
    q["t"][p["i"] < 0] = float("inf")                             # nor what stands where there is no entry
    loss2, lse2 = forward(vl, q)
    dX2, dW2 = backward(vl, q, s)
    for a, b in ((loss, loss2), (lse, lse2), (dX, dX2), (dW, dW2)):
        assert torch.equal(a, b)
    assert bool((loss[dead] == 0).all()) and bool((lse[dead] == 0).all()) and bool((dX[dead] == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [40, 200])
def test_an_entry_that_is_no_column(vl, dtype, N):
    D, V, K = 64, 300, 6
    p = batch(N, D, V, K, dtype, 12)
    p["i"][7, 3], p["i"][39, 0] = V, 2 ** 40
    ref = Reference(p)
    from paper_2405_17991_b200 import binding
    for op, call in ((vl.OP_HEAD_DISTILL, forward), (vl.OP_HEAD_DISTILL_BACKWARD, None)):
        ws = vl.velora_workspace_alloc(vl.velora_workspace_bytes(op | f32(vl, dtype), N, D, V, K), DEV)
        if call:
            loss, lse = forward(vl, p, ws=ws)
            bad = torch.isnan(loss)
            assert bad.nonzero()[:, 0].tolist() == [7, 39]
            check(loss[~bad], ref.loss[~bad], ref.loss_bound[~bad], "loss")
        else:
            dX, dW = backward(vl, p, lse, ws=ws)
            check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
            check(dW, ref.dW, ref.dW_bound, "dW", half_step(dtype))
        assert vl.velora_workspace_status(ws) == binding.ERR_INVALID_ARG
        vl.velora_workspace_init(ws)
        assert vl.velora_workspace_status(ws) == 0


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [10, 200])
def test_non_finite_logits_stay_with_their_token(vl, dtype, N, whole):
    p = batch(N, 64, 500, 5, dtype, 40, whole=whole)
    p["i"][:, 0] = torch.arange(N, device=DEV)
    loss, lse = forward(vl, p)
    p["t"][3, 0], p["t"][6, 0] = float("nan"), float("inf")
    p["X"][8, 5] = float("nan")
    loss2, lse2 = forward(vl, p)
    bad = torch.zeros(N, dtype=torch.bool, device=DEV)
    bad[3] = bad[6] = bad[8] = True
    assert bool(torch.isnan(loss2[bad]).all()) and torch.equal(loss[~bad], loss2[~bad])
    dX, _ = backward(vl, p, lse2)
    assert bool(torch.isnan(dX[bad]).any(1).all()) and bool(torch.isfinite(dX[~bad]).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V", [(1, 256, 1000), (64, 128, 3001), (200, 520, 2500)])
def test_one_entry_is_a_target(vl, dtype, N, D, V):
    """A list of one column, and lists of that column and of others without a share: the head's loss."""
    p = batch(N, D, V, 1, dtype, 30)
    p["i"] = p["i"].abs() % V
    target = p["i"][:, 0].contiguous()
    ref = Reference(p)
    want, lse0 = vl.velora_head_loss(p["X"], p["W"], target)
    more = {**p, "i": torch.cat([(p["i"] + 1) % V, p["i"], p["i"] - 2 ** 40], 1), "t": torch.cat([torch.full((N, 1), -float("inf"), device=DEV), p["t"], p["t"]], 1)}
    for q in (p, more):
        loss, lse = forward(vl, q)
        check(loss, want.double(), 2 * ref.loss_bound, "loss")
        check(lse, lse0.double(), 2 * ref.lse_bound, "lse")
        dX, dW = backward(vl, q, lse)
        dX0, dW0 = vl.velora_head_loss_backward(p["X"], p["W"], target, lse0, p["g"])
        check(dX, dX0.double(), 2 * ref.dX_bound, "dX", 2 * half_step(dtype))
        check(dW, dW0.double(), 2 * ref.dW_bound, "dW", 2 * half_step(dtype))


@pytest.mark.parametrize("N", [4, 100, 300])
def test_a_student_that_agrees(vl, N):
    """Teacher and student the same: every column's probability is the student's own share, so what is left of G = q - p is what both round by.  The
    teacher's logits are the student's, computed in fp64 and rounded to fp32: another u |l| in p."""
    D, V, K = 256, 600, 600
    p = batch(N, D, V, K, torch.bfloat16, 33)
    l = p["X"].double() @ p["W"].double().t()
    p["i"] = torch.stack([torch.randperm(V, device=DEV) for _ in range(N)])
    p["t"] = l.gather(1, p["i"]).float()
    ref = Reference(p)
    loss, lse = forward(vl, p)
    check(loss, ref.loss, ref.loss_bound, "loss")
    dX, dW = backward(vl, p, lse)
    check(dX, ref.dX, ref.dX_bound, "dX", half_step(torch.bfloat16))
    check(dW, ref.dW, ref.dW_bound, "dW", half_step(torch.bfloat16))
    q = torch.softmax(l, 1)
    assert dX.double().norm() <= 2.0 ** -12 * ((q * p["g"].double()[:, None].abs()) @ p["W"].double().abs()).norm()      # nothing near G's parts' size


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_small_workspaces_mean_smaller_pieces(vl, guard, dtype):
    N, D, V, K = 300, 136, 5000, 20
    p = batch(N, D, V, K, dtype, 50, 2.0, "some")
    ref = Reference(p)
    _, lse = forward(vl, p)
    op = vl.OP_HEAD_DISTILL_BACKWARD | f32(vl, dtype)
    full = vl.velora_workspace_bytes(op, N, D, V, K, False)
    tiny = vl.velora_workspace_bytes(op, N, D, 256, K, False) + 2 * N * ((V + 127) // 128) + 256   # a vocabulary of one piece, this one's starts
    assert tiny < full
    for size in (tiny, tiny + 2 * 256 * N * 4, full, 2 * full):
        dX, dW = backward(vl, p, lse, ws=guard.workspace(vl, size))
        check(dX, ref.dX, ref.dX_bound, "dX", half_step(dtype))
        check(dW, ref.dW, ref.dW_bound, "dW", half_step(dtype))
    with pytest.raises(vl.VeloraError):
        backward(vl, p, lse, ws=torch.zeros(4096, dtype=torch.uint8, device=DEV))
    with pytest.raises(vl.VeloraError):
        forward(vl, p, ws=torch.zeros(4096, dtype=torch.uint8, device=DEV))


def test_gradients_against_differences(vl):
    """Central differences of the loss along random directions, fp32, h = 1/64: as for the head's loss (its third derivative is log sum exp's, too)."""
    N, D, V, K = 20, 32, 60, 7
    p = batch(N, D, V, K, torch.float32, 60, 1.5, "none", True)
    p["g"] = torch.full((N,), 1.0 / N, device=DEV)
    loss, lse = forward(vl, p)
    dX, dW = backward(vl, p, lse)
    ref = Reference(p)
    err = (ref.loss_bound.max() * 1.5).item()
    gen = torch.Generator(device=DEV).manual_seed(1)
    h = 1.0 / 64
    for which, grad in (("X", dX), ("W", dW)):
        for _ in range(3):
            d = torch.randn(p[which].shape, generator=gen, device=DEV)
            d = d / d.norm()
            total = lambda s: forward(vl, {**p, which: p[which] + s * d})[0].double().mean().item()  # noqa: E731
            r = 2 * ((d @ p["W"].t()).abs().max() if which == "X" else (p["X"] @ d.t()).abs().max()).item() / p["T"]
            slope = (grad.double() * d.double()).sum().item()
            moved = 8 * U * grad.double().abs().sum().item() / h
            assert abs((total(h) - total(-h)) / (2 * h) - slope) <= h * h * r ** 3 / 3 + err / h + moved


def test_refused_on_the_card(vl):
    p = batch(6, 64, 100, 5, torch.bfloat16, 3)
    _, lse = forward(vl, p)
    for q in ({"i": p["i"].int()}, {"i": p["i"][:5]}, {"t": p["t"][:, :4]}, {"i": p["i"].t().contiguous().t()}, {"W": p["W"].float()}, {"i": p["i"].cpu()},
              {"lse": p["t"][:, 0].double()}, {"t": p["t"].half()}):
        for call in (lambda: forward(vl, {**p, **q}), lambda: backward(vl, {**p, **q}, lse)):
            with pytest.raises((ValueError, TypeError)):
                call()
    for q in ({"T": 0.0}, {"T": float("nan")}, {"i": p["i"][:1].expand(6, 5), "t": p["t"]}, {"i": torch.zeros((6, 1025), dtype=torch.int64, device=DEV), "t": torch.zeros((6, 1025), device=DEV)},
              {"i": p["i"][:, :0], "t": p["t"][:, :0]}):
        for call in (lambda: forward(vl, {**p, **q}), lambda: backward(vl, {**p, **q}, lse)):
            with pytest.raises(vl.VeloraError):
                call()


def test_empty_batch(vl):
    X, W = torch.empty((0, 64), device=DEV, dtype=torch.bfloat16), torch.randn((30, 64), device=DEV).to(torch.bfloat16)
    i, t, none = torch.empty((0, 5), dtype=torch.int64, device=DEV), torch.empty((0, 5), device=DEV), torch.empty(0, device=DEV)
    loss, lse = vl.velora_head_distill(X, W, i, t)
    assert loss.shape == (0,) and lse.shape == (0,)
    dW = torch.ones_like(W)
    vl.velora_head_distill_backward(X, W, i, t, lse, none, dW=dW, beta=1)
    assert bool((dW == 1).all())
    dX, _ = vl.velora_head_distill_backward(X, W, i, t, lse, none, dW=dW)
    assert dX.shape == (0, 64) and bool((dW == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [20, 200])
def test_captured_replayed_and_on_another_stream(vl, dtype, N):
    D, V, K = 128, 1500, 24
    first, second = (batch(N, D, V, K, dtype, s, 2.0, m, True) for s, m in ((70, "some"), (71, "none")))

    def both(p, **k):
        loss, lse = forward(vl, p, **k)
        return (loss, *backward(vl, p, lse, **k))

    want = [both(first), both(second)]
    p = {k: v.clone() if torch.is_tensor(v) else v for k, v in first.items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(p)
    for case, ref in ((second, want[1]), (first, want[0])):        # the number of tokens with entries differs from the captured one
        for k in p:
            if torch.is_tensor(p[k]):
                p[k].copy_(case[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, ref))
    outs = []
    for q in (first, second):                                     # two streams at once, a workspace each
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        outs.append(both(q, stream=s))
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lists_past_32_bits(vl, dtype):
    """Pitches that put the last tokens' lists more than 2^31 elements behind the first's."""
    N, D, V, K = 150, 64, 600, 7
    p = batch(N, D, V, K, dtype, 7, 1.0, "some", False, torch.bfloat16)
    loss, lse = forward(vl, p)
    dX, dW = backward(vl, p, lse)
    far = lambda x, shift: torch.empty_strided(x.shape, (1 << shift, 1), dtype=x.dtype, device=DEV).copy_(x)  # noqa: E731
    assert (N - 1) << 24 > 2 ** 31
    q = {**p, "i": far(p["i"], 24), "t": far(p["t"], 24)}
    loss2, lse2 = forward(vl, q)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    dX2, dW2 = backward(vl, q, lse2)
    assert torch.equal(dX, dX2) and torch.equal(dW, dW2)
