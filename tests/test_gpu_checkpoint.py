"""8-bit checkpoints of layer inputs on the GPU: codes and exponents bit for bit against the definition in 64 bits, what is read back, and
the weight gradient taken from them."""
import numpy as np
import pytest
import torch

from _util import C_SUM, TOL_GEMM, Guard, assert_matches, to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda"
BLOCK = 32


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


def definition(X: torch.Tensor):
    """(codes, exponent bytes, Xhat in 64 bits) of the definition; X on any device, the arithmetic in numpy's float64."""
    x = to_f64(X)
    N, D = x.shape
    blocks = -(-D // BLOCK)
    pad = np.zeros((N, blocks * BLOCK))
    pad[:, :D] = x
    pad = pad.reshape(N, blocks, BLOCK)
    with np.errstate(all="ignore"):
        a = np.abs(pad).max(axis=2)
        bad = ~np.isfinite(pad).all(axis=2)
        a = np.where(bad, 0.0, a)
        m, k = np.frexp(a)                                     # a = m 2^k, 1/2 <= m < 1
        e = np.where(a == 0, -126, np.clip(np.where(m * 128 <= 127, k - 7, k - 6), -126, 121))
        step = np.ldexp(1.0, e)[:, :, None]
        q = np.where(bad[:, :, None], 0.0, np.clip(np.rint(pad / step), -127, 127))
    xhat = np.where(bad[:, :, None], np.nan, q * step)
    return (q.reshape(N, -1)[:, :D].astype(np.int8), np.where(bad, 255, e + 127).astype(np.uint8), xhat.reshape(N, -1)[:, :D])


def inputs(N, D, dtype, seed, rows="padded"):
    """Heavy-tailed channels, rows of zeros, and the values that the format has to deal with planted in the first rows."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn((N, D), generator=g, device=DEV) * torch.exp(2.0 * torch.randn(D, generator=g, device=DEV))
    if N > 2:
        x[N // 2] = 0.0
    big = torch.finfo(dtype).max
    plants = [127.0, 127.5, 128.0, 0.5, 1.5, 2.5, 126.5, 2.0 ** -126, 2.0 ** -133, 1e-38, big, -big, float("inf"), float("nan"), -0.0, 127.0 * 2.0 ** 100]
    for i, p in enumerate(plants):
        if i < N:
            x[i, (7 * i) % D] = p
            x[i, (7 * i + 1) % D] = p / 3 if abs(p) < 1e30 else 1.0
    x = x.to(dtype)
    if rows == "dense":
        return x.contiguous()
    ld = -(-D // 8) * 8 + (8 if rows == "padded" else 9)       # 9: rows on odd boundaries
    buf = torch.zeros((N, ld + 1), dtype=dtype, device=DEV) if rows == "offset" else torch.zeros((N, ld), dtype=dtype, device=DEV)
    view = buf[:, 1:1 + D] if rows == "offset" else buf[:, :D]
    view.copy_(x)
    return view


def equal_values(got: torch.Tensor, ref: np.ndarray):
    g = to_f64(got)
    assert np.array_equal(np.isnan(g), np.isnan(ref))
    assert np.array_equal(np.nan_to_num(g), np.nan_to_num(ref))


SIZES = [(1, 1), (3, 1), (20, 1), (9, 3), (1, 31), (3, 32), (2, 33), (5, 255), (4, 257), (7, 1000), (40, 264), (64, 4096), (33, 5461), (20000, 64), (3000, 520)]


@pytest.mark.parametrize("rows", ["padded", "dense", "offset"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D", SIZES)
def test_codes_exponents_and_what_is_read_back(vl, guard, N, D, dtype, rows):
    X = inputs(N, D, dtype, 100 * N + D, rows)
    q_ref, e_ref, xhat = definition(X)
    # codes and exponents with guard bands; pitches that are and are not multiples of 8
    Q = guard.mat(N, D, torch.uint8, ld=None if rows == "padded" else D + 3).view(torch.int8)
    E = guard.mat(N, -(-D // BLOCK), torch.uint8, ld=None if rows == "padded" else -(-D // BLOCK) + 1)
    out = vl.velora_checkpoint_store(X, Q, E)
    assert out[0] is Q and out[1] is E
    assert np.array_equal(Q.cpu().numpy(), q_ref)
    assert np.array_equal(E.cpu().numpy(), e_ref)
    for out_dtype in (torch.bfloat16, torch.float32):
        back = guard.mat(N, D, out_dtype, ld=None if rows == "padded" else D + 1)
        vl.velora_checkpoint_load(Q, E, back)
        equal_values(back, xhat)
    # with buffers of the binding's own
    Q2, E2 = vl.velora_checkpoint_store(X)
    assert torch.equal(Q2, Q) and torch.equal(E2, E)
    equal_values(vl.velora_checkpoint_load(Q2, E2, x_dtype=dtype), xhat)


def test_error_is_half_a_step(vl):
    """|Xhat - X| <= s / 2 and s < 2 a / 127, so at most a / 127 of the block's largest value."""
    X = torch.randn((512, 1024), device=DEV, generator=torch.Generator(device=DEV).manual_seed(5))
    Q, E = vl.velora_checkpoint_store(X)
    back = vl.velora_checkpoint_load(Q, E, x_dtype=torch.float32)
    a = X.view(512, -1, BLOCK).abs().amax(2, keepdim=True)
    assert bool(((back - X).view(512, -1, BLOCK).abs() <= a / 127 * (1 + 2 ** -20)).all())
    assert int(Q.to(torch.int32).abs().max()) <= 127
    # a checkpoint of what was read back is the same checkpoint's values
    Q3, E3 = vl.velora_checkpoint_store(back)
    assert torch.equal(vl.velora_checkpoint_load(Q3, E3, x_dtype=torch.float32), back)


def finite_inputs(N, D, O, dtype, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    X = (torch.randn((N, D), generator=g, device=DEV) * torch.exp(0.5 * torch.randn(D, generator=g, device=DEV))).to(dtype)
    dY = torch.randn((N, O), generator=g, device=DEV).to(dtype)
    return X, dY


GRADS = [(1, 32, 8), (3, 8, 8), (17, 40, 24), (64, 128, 128), (65, 136, 264), (200, 77, 45), (1000, 512, 1376), (4096, 512, 512), (2049, 1376, 512),
         (333, 1000, 2048), (8192, 1024, 1024), (4104, 2056, 2056), (700, 5461, 520)]


@pytest.mark.parametrize("dtype,dw_dtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32),
                                            (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("N,D,O", GRADS)
def test_weight_grad(vl, guard, N, D, O, dtype, dw_dtype):
    X, dY = finite_inputs(N, D, O, dtype, N + D + O)
    Q, E = vl.velora_checkpoint_store(X)
    xhat = torch.from_numpy(definition(X)[2]).to(DEV)
    ref = dY.double().t() @ xhat
    op = vl.OP_CHECKPOINT_WEIGHT_GRAD | (vl.OP_F32 if dtype == torch.float32 else 0)
    for ld, any_rows in ((None, True), (D, False)):
        dW = guard.mat(O, D, dw_dtype, ld=ld)
        ws = guard.workspace(vl, vl.velora_workspace_bytes(op, N, D, O, 1, any_rows))
        vl.velora_checkpoint_weight_grad(dY, Q, E, dW, ws=ws)
        assert_matches(dW, ref.cpu().numpy(), TOL_GEMM, "dW", c=C_SUM)
        assert vl.velora_workspace_status(ws) == 0
    # beta = 1 adds to what is there
    start = torch.randn((O, D), device=DEV).to(dw_dtype)
    dW = guard.mat(O, D, dw_dtype, init=start)
    vl.velora_checkpoint_weight_grad(dY, Q, E, dW, beta=1)
    assert_matches(dW, (ref + start.double()).cpu().numpy(), TOL_GEMM, "dW, beta = 1", c=C_SUM)


@pytest.mark.parametrize("N,D,O", [(200, 264, 520), (1500, 1032, 2056)])
def test_weight_grad_of_views_on_any_boundary(vl, guard, N, D, O):
    """Codes, exponents and dY as views that start and step anywhere give what aligned ones give."""
    X, dY = finite_inputs(N, D, O, torch.bfloat16, 3)
    Q, E = vl.velora_checkpoint_store(X)
    ref = (dY.double().t() @ torch.from_numpy(definition(X)[2]).to(DEV)).cpu().numpy()

    def moved(t, left, right):
        buf = torch.full((t.shape[0], t.shape[1] + left + right), 77, device=DEV, dtype=t.dtype)
        buf[:, left:left + t.shape[1]] = t
        return buf[:, left:left + t.shape[1]]

    for q, e, y in ((moved(Q, 1, 2), E, dY), (Q, moved(E, 1, 0), dY), (moved(Q, 16, 8), moved(E, 4, 3), moved(dY, 8, 0)), (moved(Q, 3, 0), moved(E, 2, 1), moved(dY, 1, 0))):
        dW = guard.mat(O, D)
        vl.velora_checkpoint_weight_grad(y, q, e, dW)
        assert_matches(dW, ref, TOL_GEMM, "dW", c=C_SUM)


def test_a_block_with_a_nan_reaches_its_columns_alone(vl):
    N, D, O = 300, 320, 264
    X, dY = finite_inputs(N, D, O, torch.bfloat16, 9)
    X[17, 70] = float("nan")
    X[250, 319] = float("inf")
    Q, E = vl.velora_checkpoint_store(X)
    dW = vl.velora_checkpoint_weight_grad(dY, Q, E)
    hit = torch.zeros(D, dtype=torch.bool, device=DEV)
    hit[64:96] = True
    hit[288:320] = True
    assert bool(torch.isnan(dW[:, hit]).all()) and bool(torch.isfinite(dW[:, ~hit]).all())


def test_empty_batch(vl):
    Q, E = vl.velora_checkpoint_store(torch.empty((0, 40), device=DEV, dtype=torch.bfloat16))
    assert Q.shape == (0, 40) and E.shape == (0, 2)
    assert vl.velora_checkpoint_load(Q, E).shape == (0, 40)
    dY = torch.empty((0, 24), device=DEV, dtype=torch.bfloat16)
    dW = torch.ones((24, 40), device=DEV, dtype=torch.bfloat16)
    vl.velora_checkpoint_weight_grad(dY, Q, E, dW, beta=1)
    assert bool((dW == 1).all())
    vl.velora_checkpoint_weight_grad(dY, Q, E, dW)
    assert bool((dW == 0).all())


def test_offsets_past_32_bits(vl):
    """70000 rows with a pitch of 65536 bytes: codes lie past 2^32."""
    N, D, ld = 70000, 96, 65536
    buf = torch.zeros(N * ld, dtype=torch.int8, device=DEV)
    Q = buf.view(N, ld)[:, :D]
    X = torch.randn((N, D), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(torch.bfloat16)
    E = torch.empty((N, 3), dtype=torch.uint8, device=DEV)
    vl.velora_checkpoint_store(X, Q, E)
    Q2, E2 = vl.velora_checkpoint_store(X)
    assert torch.equal(Q.contiguous(), Q2.contiguous()) and torch.equal(E, E2.contiguous())
    assert torch.equal(vl.velora_checkpoint_load(Q, E), vl.velora_checkpoint_load(Q2, E2))
    dY = torch.randn((N, 264), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)).to(torch.bfloat16)
    assert torch.equal(vl.velora_checkpoint_weight_grad(dY, Q, E), vl.velora_checkpoint_weight_grad(dY, Q2, E2))


@pytest.mark.parametrize("N,D,O", [(777, 1032, 520), (4096, 2048, 2048)])
def test_captured_replayed_and_on_another_stream(vl, N, D, O):
    """Store and weight gradient from a graph, on inputs that change between replays, and on a side stream: the same bits."""
    X, dY = finite_inputs(N, D, O, torch.bfloat16, 21)
    X2, dY2 = finite_inputs(N, D, O, torch.bfloat16, 22)
    ws = vl.velora_workspace_alloc(vl.velora_workspace_bytes(vl.OP_CHECKPOINT_WEIGHT_GRAD, N, D, O, 1), DEV)
    Q, E = vl.velora_checkpoint_store(X)
    dW = vl.velora_checkpoint_weight_grad(dY, Q, E, ws=ws)
    want = [dW.clone()]
    Q2, E2 = vl.velora_checkpoint_store(X2)
    want.append(vl.velora_checkpoint_weight_grad(dY2, Q2, E2).clone())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            vl.velora_checkpoint_store(X, Q, E)
            vl.velora_checkpoint_weight_grad(dY, Q, E, dW, ws=ws)
    first = (X.clone(), dY.clone())
    for x, y, w in ((*first, want[0]), (X2, dY2, want[1]), (*first, want[0])):
        X.copy_(x)
        dY.copy_(y)
        dW.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dW, w)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    q, e = vl.velora_checkpoint_store(X2, stream=other)
    got = vl.velora_checkpoint_weight_grad(dY2, q, e, ws=torch.zeros_like(ws), stream=other)
    other.synchronize()
    assert torch.equal(got, want[1])


def test_weight_grad_refuses_a_workspace_without_room(vl):
    N, D, O = 64, 128, 128
    X, dY = finite_inputs(N, D, O, torch.bfloat16, 7)
    Q, E = vl.velora_checkpoint_store(X)
    with pytest.raises(vl.VeloraError):
        vl.velora_checkpoint_weight_grad(dY, Q, E, ws=vl.velora_workspace_alloc(256, DEV))


@pytest.mark.parametrize("dw_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,O,padded", [(8200, 2304, 2304, True), (8200, 2303, 2305, False), (9001, 4096, 1300, True)])
def test_weight_grad_whose_last_wave_is_cut(vl, guard, N, D, O, padded, dw_dtype):
    """Tiles of 256 x 256 on 74 pairs: 81, 90, 96, so the last wave's 7, 16 or 22 are cut into 8, 4 or 3 parts of the contraction.  Whatever
    stands in the workspace, twice the same bits, beta = 1, and the uncut product of a workspace without the room."""
    X, dY = finite_inputs(N, D, O, torch.bfloat16, N + D + O)
    Q, E = vl.velora_checkpoint_store(X)
    ref = dY.double().t() @ vl.velora_checkpoint_load(Q, E, x_dtype=torch.float32).double()
    size = vl.velora_workspace_bytes(vl.OP_CHECKPOINT_WEIGHT_GRAD, N, D, O, 1, not padded)
    assert size > 256 + 2 * N * (D + 7) + (0 if padded else 2 * N * (O + 7)) + (10 << 20)
    got = []
    for fill in (0, 255):
        ws = guard.workspace(vl, size)
        ws[256:] = fill
        dW = guard.mat(O, D, dw_dtype, ld=None if padded else D)
        vl.velora_checkpoint_weight_grad(dY, Q, E, dW, ws=ws)
        assert_matches(dW, ref.cpu().numpy(), TOL_GEMM, "dW", c=C_SUM)
        vl.velora_checkpoint_weight_grad(dY, Q, E, dW, ws=ws)
        assert vl.velora_workspace_status(ws) == 0
        got.append(dW.clone())
    assert torch.equal(got[0], got[1])
    start = torch.randn((O, D), device=DEV).to(dw_dtype)
    dW = guard.mat(O, D, dw_dtype, init=start)
    vl.velora_checkpoint_weight_grad(dY, Q, E, dW, beta=1)
    assert_matches(dW, (ref + start.double()).cpu().numpy(), TOL_GEMM, "dW, beta = 1", c=C_SUM)
    less = guard.workspace(vl, size - 256)
    dW = guard.mat(O, D, dw_dtype)
    vl.velora_checkpoint_weight_grad(dY, Q, E, dW, ws=less)
    assert_matches(dW, ref.cpu().numpy(), TOL_GEMM, "dW, uncut", c=C_SUM)
