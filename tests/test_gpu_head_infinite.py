"""Logits of minus infinity (a column that a sum past the type's range takes out): such a column has no share, wherever it stands in the vocabulary."""
import pytest
import torch

from test_gpu_head_loss import Reference, check

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def vl():
    import paper_2405_17991_b200 as pkg
    pkg.lib()
    return pkg


@pytest.mark.parametrize("where", ["first", "middle", "last", "all but one"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V", [(7, 64, 1000), (40, 64, 1000), (300, 256, 2049)])
def test_columns_of_minus_infinity(vl, N, D, V, dtype, where):
    """Pieces of 256 columns (fp32), segments of 128 (bf16), whole ones of them at minus infinity."""
    g = torch.Generator(device=DEV)
    g.manual_seed(N + V)
    X = torch.randn((N, D), generator=g, device=DEV)
    X[:, 0] = 4.0
    W = torch.randn((V, D), generator=g, device=DEV) / D ** 0.5
    gone = torch.zeros(V, dtype=torch.bool, device=DEV)
    gone[{"first": slice(0, 512), "middle": slice(256, 520), "last": slice(V - 500, V), "all but one": slice(0, V - 1)}[where]] = True
    left = (~gone).nonzero()[:, 0]
    t = left[torch.randint(left.shape[0], (N,), generator=g, device=DEV)]
    X, W = X.to(dtype), W.to(dtype)
    W[gone, 0] = -3e38                                             # 4 times that is past the range
    ref = Reference(X, W[left], torch.searchsorted(left, t), torch.ones(N, device=DEV))
    f32 = vl.OP_F32 if dtype == torch.float32 else 0
    for columns in (256, V):                                       # room for one piece of 256 columns; for all there are
        ws = vl.velora_workspace_alloc(max(vl.velora_workspace_bytes(vl.OP_HEAD_LOSS | f32, N, D, columns, 1, False),
                                           vl.velora_workspace_bytes(vl.OP_HEAD_LOSS, N, D, V, 1, False) if not f32 else 0), DEV)
        loss, lse = vl.velora_head_loss(X, W, t, ws=ws)
        check(loss, ref.loss, ref.loss_bound, "loss", 0)
        check(lse, ref.lse, ref.loss_bound, "lse", 0)
