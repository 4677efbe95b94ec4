"""Layer norm and its gradients on the GPU against the formula in 64 bits.

Bounds, element by element, u = 2^-24.  A sum of D values over a row is a tree whose branches are at most L = 32 + D / 256 additions deep (a thread's own
values, a warp's, the block's), so it is off by L u times the sum of sizes.
  m      e = L u mean|h| + u |m|
  var    (h - m rounds by u |h - m|, a shift of m by e adds e^2): e^2 + (L + 4) u var;    r: half of that relative to var + eps, and 3u
  xhat   (e + 2u |h - m|) r + |xhat| (r's)
  y      |w| (xhat's) + 3u (|xhat w| + |b|), and half a step of the output's type
Backward pass, from the fp32 m and r as given: xhat and c are off by 3u of themselves, their means by L u of the sums of sizes besides;
  dx     r (4u |c| + mean's + |xhat| mean's + 6u |xhat mean(c xhat)|) + 2u (|dh| + |dx|), and half a step
  dw, db sums over the rows in branches of at most 64 + N / 100 additions: (64 + N / 100 + 4) u sum |dy xhat|, and half a step of their type
"""
import pytest
import torch

from _util import Guard

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
EPS = 1e-5


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


def depth(D):
    return 32 + D / 256


def batch(N, D, dtype, seed, p_dtype=torch.float32, offset=0.0, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    X = ((r(N, D) * torch.exp(0.5 * r(D)) + offset) * scale).to(dtype)
    return {"X": X, "R": (r(N, D) * scale).to(dtype), "w": (1 + 0.3 * r(D)).to(p_dtype), "b": (0.5 * r(D)).to(p_dtype), "dY": r(N, D).to(dtype), "dH": r(N, D).to(dtype)}


class Forward:
    def __init__(self, X, R, w, b, eps=EPS):
        D, dtype = X.shape[1], X.dtype
        self.H = X if R is None else (X.float() + R.float()).to(dtype)
        h = self.H.double()
        w = torch.ones(D, device=DEV, dtype=torch.float64) if w is None else w.double()
        b = torch.zeros(D, device=DEV, dtype=torch.float64) if b is None else b.double()
        L = depth(D)
        self.m = h.mean(1)
        self.m_bound = L * U * h.abs().mean(1) + U * self.m.abs()
        c = h - self.m[:, None]
        var = (c * c).mean(1)
        self.r = 1 / torch.sqrt(var + eps)
        rel = (self.m_bound ** 2 + (L + 4) * U * var) / (var + eps) / 2 + 3 * U
        self.r_bound = rel * self.r
        xhat = c * self.r[:, None]
        dx = (self.m_bound[:, None] + 2 * U * c.abs()) * self.r[:, None] + xhat.abs() * rel[:, None]
        self.Y = xhat * w + b
        self.Y_bound = w.abs() * dx + 3 * U * ((xhat * w).abs() + b.abs())


class Backward:
    def __init__(self, dY, H, mean, rstd, w, dH):
        N, D = H.shape
        dy, r = dY.double(), rstd.double()[:, None]
        w = torch.ones(D, device=DEV, dtype=torch.float64) if w is None else w.double()
        xhat = (H.double() - mean.double()[:, None]) * r
        c = dy * w
        a, b = c.mean(1, keepdim=True), (c * xhat).mean(1, keepdim=True)
        da = (depth(D) + 3) * U * c.abs().mean(1, keepdim=True)
        db = (depth(D) + 6) * U * (c * xhat).abs().mean(1, keepdim=True)
        self.dX = r * (c - a - xhat * b)
        self.dX_bound = r * (4 * U * c.abs() + da + 2 * U * a.abs() + xhat.abs() * db + 6 * U * (xhat * b).abs()) + 2 * U * self.dX.abs()
        if dH is not None:
            self.dX = self.dX + dH.double()
            self.dX_bound = self.dX_bound + 2 * U * dH.double().abs()
        rows = (64 + N / 100 + 4) * U
        self.dw, self.db = (dy * xhat).sum(0), dy.sum(0)
        self.dw_bound, self.db_bound = rows * (dy * xhat).abs().sum(0), rows * dy.abs().sum(0)


def check(got, ref, bound, what, rounding=0.0):
    assert bool(torch.isfinite(got).all()), what
    bound = bound + (rounding + U) * ref.abs() + 1e-30
    diff = (got.double() - ref).abs()
    worst = (diff / bound).max().item() if diff.numel() else 0.0
    assert worst <= 1.0, "%s: %.3g times its bound" % (what, worst)


def run(vl, guard, p, residual, dtype, dw_dtype=torch.float32, ld=None, w=True, b=True):
    """Both passes into guarded outputs, each checked."""
    N, D = p["X"].shape
    mat = lambda: guard.mat(N, D, dtype, ld=ld)  # noqa: E731
    R, weight, bias = p["R"] if residual else None, p["w"] if w else None, p["b"] if b else None
    ref = Forward(p["X"], R, weight, bias)
    Y, H, mean, rstd = vl.velora_layer_norm(p["X"], weight, bias, EPS, R, mat(), mat() if residual else None, guard.vec(N), guard.vec(N))
    assert torch.equal(H, ref.H)
    check(mean, ref.m, ref.m_bound, "mean")
    check(rstd, ref.r, ref.r_bound, "rstd")
    check(Y, ref.Y, ref.Y_bound, "Y", half_step(dtype))
    dH = p["dH"] if residual else None
    back = Backward(p["dY"], H, mean, rstd, weight, dH)
    ws = guard.workspace(vl, vl.velora_workspace_bytes(vl.OP_LAYER_NORM_BACKWARD, N, D, 1, 1, False))
    dX, dw, db = vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, weight, dH, mat(), guard.vec(D, dw_dtype), guard.vec(D, dw_dtype), ws=ws)
    check(dX, back.dX, back.dX_bound, "dX", half_step(dtype))
    check(dw, back.dw, back.dw_bound, "dweight", half_step(dw_dtype))
    check(db, back.db, back.db_bound, "dbias", half_step(dw_dtype))
    return Y, H, mean, rstd, dX, dw, db


SIZES = [(1, 1), (1, 2), (3, 7), (1, 8), (5, 33), (1, 64), (2, 256), (9, 257), (300, 512), (17, 520), (1000, 768), (31, 1000), (7, 1024), (70, 1032), (150, 2048),
         (1, 4096), (200, 4096), (33, 5461), (20, 6145), (640, 8), (15, 8192), (9, 11008), (3, 12290), (2, 16384), (3, 16400), (2, 40001)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D", SIZES)
def test_norm_and_gradients(vl, guard, N, D, dtype, residual):
    """Rows on 16-byte boundaries with padding, then dense rows."""
    p = batch(N, D, dtype, N + D, dtype if residual else torch.float32)
    run(vl, guard, p, residual, dtype, dw_dtype=dtype)
    run(vl, guard, p, residual, dtype, ld=D)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
def test_widths_around_every_multiple_of_a_warps_words(vl, guard, dtype, residual):
    """Rows of 32 n - 1, 32 n and 32 n + 1 words of 16 bytes, up to the longest that is held and beyond."""
    words = torch.finfo(dtype).bits // 8
    per = 16 // words
    for n in list(range(1, 12)) + list(range(13, 16)) + list(range(16, 98, 3)):
        for w in (32 * n - 1, 32 * n, 32 * n + 1):
            run(vl, guard, batch(2, w * per, dtype, w), residual, dtype)


@pytest.mark.parametrize("residual", [False, True])
def test_odd_widths_around_every_tier(vl, guard, residual):
    for D in (31, 33, 255, 257, 511, 513, 1023, 1025, 2047, 2049, 2559, 2561, 4095, 4097, 5631, 5633, 7167, 7169, 8191, 8193, 10239, 10241, 12287, 12289):
        run(vl, guard, batch(5, D, torch.bfloat16, D), residual, torch.bfloat16, ld=D)
        if D % 4 == 1:
            run(vl, guard, batch(3, D, torch.float32, D), residual, torch.float32, ld=D)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("D,dtype", [(8200, torch.bfloat16), (11008, torch.bfloat16), (12288, torch.bfloat16), (4100, torch.float32), (5464, torch.float32), (6144, torch.float32)])
def test_blocks_of_two_rows_and_more(vl, guard, D, dtype, residual):
    """Numbers of rows that give blocks 1, 2, 3 or 9 rows, or both of two neighbouring numbers; each row as it is by itself, and in place."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for N in (sms - 1, sms + 7, 2 * sms, 3 * sms, 3 * sms + 1, 9 * sms):
        p = batch(N, D, dtype, N)
        Y, _, mean, rstd = run(vl, guard, p, residual, dtype)[:4]
        for i in (0, N // 2, N - 1):
            one = vl.velora_layer_norm(p["X"][i:i + 1], p["w"], p["b"], EPS, p["R"][i:i + 1] if residual else None)
            assert torch.equal(one[0][0], Y[i]) and torch.equal(one[2][0], mean[i]) and torch.equal(one[3][0], rstd[i])
        vl.velora_layer_norm(p["X"], p["w"], p["b"], EPS, p["R"] if residual else None, Y=p["X"], H=None if not residual else p["R"])
        assert torch.equal(p["X"], Y)


def test_more_rows_than_slices_or_blocks(vl, guard):
    for N, D in ((20011, 24), (5003, 264), (3001, 1320)):
        run(vl, guard, batch(N, D, torch.bfloat16, 3), True, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D", [(40, 768), (40, 1001), (30, 2052), (12, 4100)])
def test_rows_anywhere(vl, guard, N, D, dtype):
    """Views that start on any element, pitches that put rows on every boundary in turn, each operand's another."""
    p = batch(N, D, dtype, 5)

    def moved(x, before, after):
        buf = torch.full((N, D + before + after), float("nan"), device=DEV, dtype=dtype)
        buf[:, before:before + D] = x
        return buf[:, before:before + D]

    views = {k: moved(p[k], 1 + i, 2 * i) for i, k in enumerate(("X", "R", "dY", "dH"))}
    for keys in (("X",), ("R",), ("dY",), ("dH",), ("X", "R", "dY", "dH")):
        for ld in (None, D, D + 3):
            run(vl, guard, {**p, **{k: views[k] for k in keys}}, True, dtype, ld=ld)


@pytest.mark.parametrize("N,D", [(50, 768), (20, 4096), (6, 16400), (21, 1001)])
def test_without_weight_bias_or_some_gradients(vl, guard, N, D):
    p = batch(N, D, torch.bfloat16, 6)
    for w in (False, True):
        for b in (False, True):
            run(vl, guard, p, False, torch.bfloat16, w=w, b=b)
    Y, H, mean, rstd = vl.velora_layer_norm(p["X"], p["w"], p["b"])
    full = vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, p["w"])
    assert full[1].dtype == torch.float32
    for needs in ((True, True, False), (True, False, True), (False, True, True), (True, False, False), (False, True, False), (False, False, True)):
        some = vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, p["w"], need_dX=needs[0], need_dweight=needs[1], need_dbias=needs[2])
        for x, y, need in zip(some, full, needs):
            assert x is None if not need else torch.equal(x, y)
    assert vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, need_dX=False, need_dweight=False, need_dbias=False) == (None, None, None)


@pytest.mark.parametrize("p_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D", [(9, 64), (30, 768), (20, 4096), (9, 5461), (5, 11008), (3, 16400)])
def test_weights_and_their_gradients_anywhere(vl, guard, N, D, p_dtype):
    """Vectors that start on any element."""
    p = batch(N, D, torch.bfloat16, 8, p_dtype)
    off = lambda x, k: torch.cat([torch.full((k,), float("nan"), device=DEV, dtype=x.dtype), x])[k:]  # noqa: E731
    want = vl.velora_layer_norm(p["X"], p["w"], p["b"], residual=p["R"])
    back = vl.velora_layer_norm_backward(p["dY"], *want[1:], p["w"], dH=p["dH"])
    for k in (1, 3):
        w, b = off(p["w"], k), off(p["b"], k + 1)
        got = vl.velora_layer_norm(p["X"], w, b, residual=p["R"])
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        dw, db = (off(torch.empty_like(w), j) for j in (k, k + 1))
        got = vl.velora_layer_norm_backward(p["dY"], *got[1:], w, dH=p["dH"], dweight=dw, dbias=db)
        assert all(torch.equal(x, y) for x, y in zip(got, back))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D", [(1, 96), (77, 513), (600, 2048), (4, 20000)])
def test_gradients_are_added(vl, guard, N, D, dtype):
    p = batch(N, D, torch.bfloat16, 9)
    _, H, mean, rstd = vl.velora_layer_norm(p["X"], p["w"], p["b"])
    back = Backward(p["dY"], H, mean, rstd, p["w"], None)
    start = torch.randn(2, D, device=DEV).to(dtype)
    dw, db = start[0].clone(), start[1].clone()
    vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, p["w"], dweight=dw, dbias=db, beta=1)
    check(dw, back.dw + start[0].double(), back.dw_bound + 2 * U * start[0].double().abs(), "dweight", half_step(dtype))
    check(db, back.db + start[1].double(), back.db_bound + 2 * U * start[1].double().abs(), "dbias", half_step(dtype))
    with pytest.raises(ValueError):
        vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, p["w"], beta=1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D", [(40, 768), (40, 1001), (25, 4096), (6, 11008), (3, 16400)])
def test_outputs_in_place(vl, N, D, dtype):
    """H and Y where X or R is, dX where dY, dH or H is: the bits of outputs of their own."""
    p = batch(N, D, dtype, 10)
    want = vl.velora_layer_norm(p["X"], p["w"], p["b"], residual=p["R"])
    for h_at, y_at in (("X", "R"), ("R", "X"), ("X", None), (None, "X"), (None, "R")):
        q = {k: v.clone() for k, v in p.items()}
        H, Y = (torch.empty_like(p["X"]) if k is None else q[k] for k in (h_at, y_at))
        got = vl.velora_layer_norm(q["X"], p["w"], p["b"], residual=q["R"], Y=Y, H=H)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), (h_at, y_at)
    X = p["X"].clone()
    vl.velora_layer_norm(X, p["w"], p["b"], Y=X)
    assert torch.equal(X, vl.velora_layer_norm(p["X"], p["w"], p["b"])[0])
    Y, H, mean, rstd = want
    want = vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, p["w"], dH=p["dH"])
    for at in ("dY", "dH", "H"):
        q = {"dY": p["dY"].clone(), "dH": p["dH"].clone(), "H": H.clone()}
        got = vl.velora_layer_norm_backward(q["dY"], q["H"], mean, rstd, p["w"], dH=q["dH"], dX=q[at])
        assert all(torch.equal(x, y) for x, y in zip(got, want)), at


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [100, 1024, 4096, 16400])
def test_hard_rows(vl, dtype, D):
    """Rows far from zero, one element far from the others, all alike, zeros, very large and very small ones."""
    g = torch.Generator(device=DEV).manual_seed(4)
    r = torch.randn((8, D), generator=g, device=DEV)
    r[0] += 1000.0
    r[1, 0] = 30000.0
    r[2] = 3.0
    r[3] = 0.0
    r[4] *= 1e15
    r[5] *= 1e-15
    r[6] = -7e4
    r[6, D - 1] = 7e4
    X = r.to(dtype)
    ref = Forward(X, None, None, None)
    Y, _, mean, rstd = vl.velora_layer_norm(X)
    check(mean, ref.m, ref.m_bound, "mean")
    check(rstd, ref.r, ref.r_bound, "rstd")
    check(Y, ref.Y, ref.Y_bound, "Y", half_step(dtype))
    dY = torch.randn((8, D), generator=g, device=DEV).to(dtype)
    dX, dw, db = vl.velora_layer_norm_backward(dY, X, mean, rstd)
    back = Backward(dY, X, mean, rstd, None, None)
    check(dX, back.dX, back.dX_bound, "dX", half_step(dtype))
    check(dw, back.dw, back.dw_bound, "dweight")
    # without eps a row of equal values has nothing to be scaled by
    ref = Forward(X[4:6], None, None, None, eps=0.0)
    check(vl.velora_layer_norm(X[4:6], eps=0.0)[0], ref.Y, ref.Y_bound, "Y without eps", half_step(dtype))


@pytest.mark.parametrize("D", [96, 768, 1001, 4096, 16400])
def test_non_finite_rows_stay_by_themselves(vl, D):
    p = batch(20, D, torch.bfloat16, 13)
    clean = vl.velora_layer_norm(p["X"], p["w"], p["b"])
    X = p["X"].clone()
    X[3, D // 2], X[11, 0] = float("nan"), float("inf")
    Y, H, mean, rstd = vl.velora_layer_norm(X, p["w"], p["b"])
    bad = torch.zeros(20, dtype=torch.bool, device=DEV)
    bad[3] = bad[11] = True
    assert bool(torch.isnan(Y[bad]).all()) and torch.equal(Y[~bad], clean[0][~bad])
    dX = vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, p["w"])[0]
    assert bool(torch.isnan(dX[bad]).all()) and bool(torch.isfinite(dX[~bad]).all())


def test_derivatives_against_differences(vl):
    """Central differences of sum(dY Y) + sum(dH H) along random directions, fp32, h = 2^-6 of inputs whose rows have a deviation near 1: the third
    derivative along a unit direction is below 30 |dY w| a row, the loss's own rounding 2^-20 of its terms' sizes."""
    N, D = 12, 48
    p = batch(N, D, torch.float32, 14)
    Y, H, mean, rstd = vl.velora_layer_norm(p["X"], p["w"], p["b"], residual=p["R"])
    dX, dw, db = vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, p["w"], dH=p["dH"])
    g = torch.Generator(device=DEV).manual_seed(2)
    h = 2.0 ** -6
    size = ((p["dY"].double() * Y.double()).abs().sum() + (p["dH"].double() * H.double()).abs().sum()).item()
    third = 30 * (p["dY"].double() * p["w"].double()).norm(dim=1).sum().item() * rstd.double().max().item() ** 3
    for which, grad in (("X", dX), ("R", dX), ("w", dw), ("b", db)):
        for _ in range(3):
            d = torch.randn(p[which].shape, generator=g, device=DEV)
            d = d / d.norm()

            def total(s):
                q = {**p, which: p[which] + s * d}
                y, hh, _, _ = vl.velora_layer_norm(q["X"], q["w"], q["b"], residual=q["R"])
                return ((p["dY"].double() * y.double()).sum() + (p["dH"].double() * hh.double()).sum()).item()

            slope = (grad.double() * d.double()).sum().item()
            moved = 8 * U * grad.double().abs().sum().item() / h
            assert abs((total(h) - total(-h)) / (2 * h) - slope) <= h * h * third / 6 + 2.0 ** -20 * size / h + moved, which


def test_empty_batch(vl):
    X = torch.empty((0, 64), device=DEV, dtype=torch.bfloat16)
    w = torch.ones(64, device=DEV)
    Y, H, mean, rstd = vl.velora_layer_norm(X, w, w, residual=X)
    assert Y.shape == H.shape == (0, 64) and mean.shape == rstd.shape == (0,)
    dw, db = torch.ones(64, device=DEV), torch.ones(64, device=DEV)
    vl.velora_layer_norm_backward(Y, H, mean, rstd, w, dweight=dw, dbias=db, beta=1)
    assert bool((dw == 1).all()) and bool((db == 1).all())
    vl.velora_layer_norm_backward(Y, H, mean, rstd, w, dweight=dw, dbias=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("N,shift", [(100, 25)])
@pytest.mark.parametrize("D", [64, 1001])
def test_rows_past_32_bits(vl, N, shift, D):
    """Pitches that put the last rows more than 2^31 elements behind the first."""
    p = batch(N, D, torch.bfloat16, 7)
    far = lambda: torch.empty_strided((N, D), (1 << shift, 1), dtype=torch.bfloat16, device=DEV)  # noqa: E731
    X, H, dX = far(), far(), far()
    X.copy_(p["X"])
    want = vl.velora_layer_norm(p["X"], p["w"], p["b"], residual=p["R"])
    got = vl.velora_layer_norm(X, p["w"], p["b"], residual=p["R"], H=H, Y=X)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    want = vl.velora_layer_norm_backward(p["dY"], want[1], want[2], want[3], p["w"], dH=p["dH"])
    got = vl.velora_layer_norm_backward(p["dY"], H, got[2], got[3], p["w"], dH=p["dH"], dX=dX)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_refused_on_the_card(vl):
    p = batch(4, 64, torch.bfloat16, 1)
    for call in (lambda: vl.velora_layer_norm(p["X"], p["w"][:63]), lambda: vl.velora_layer_norm(p["X"], p["w"], p["b"].bfloat16()),
                 lambda: vl.velora_layer_norm(p["X"], residual=p["R"].float()), lambda: vl.velora_layer_norm(p["X"].t()),
                 lambda: vl.velora_layer_norm(p["X"], H=p["R"]),
                 lambda: vl.velora_layer_norm_backward(p["dY"][:3], p["X"], p["w"], p["w"])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(vl.VeloraError):
        vl.velora_layer_norm(p["X"], eps=-1.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D", [(300, 768), (100, 4096)])
def test_captured_replayed_and_on_another_stream(vl, N, D, dtype):
    first, second = batch(N, D, dtype, 70), batch(N, D, dtype, 71)

    def both(p, **out):
        Y, H, mean, rstd = vl.velora_layer_norm(p["X"], p["w"], p["b"], residual=p["R"])
        return (Y, *vl.velora_layer_norm_backward(p["dY"], H, mean, rstd, p["w"], dH=p["dH"]))

    want = [both(first), both(second)]
    p = {k: v.clone() for k, v in first.items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(p)
    for case, ref in ((second, want[1]), (first, want[0])):
        for k in p:
            p[k].copy_(case[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, ref))
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s, q in zip(streams, (first, second)):
        s.wait_stream(torch.cuda.current_stream())
        Y, H, mean, rstd = vl.velora_layer_norm(q["X"], q["w"], q["b"], residual=q["R"], stream=s)
        outs.append((Y, *vl.velora_layer_norm_backward(q["dY"], H, mean, rstd, q["w"], dH=q["dH"], stream=s)))
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
