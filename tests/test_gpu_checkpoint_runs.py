"""8-bit checkpoints in the form that wide and long inputs take: runs of four segments of 256 columns."""
import numpy as np
import pytest
import torch

from _util import Guard
from test_gpu_checkpoint import BLOCK, DEV, definition, equal_values, inputs

pytestmark = pytest.mark.gpu


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


# Four segments a run where the runs still give each of 148 x 5 x 8 warps one.  Segments, runs, what the last run has: 4, 1, whole with 9 columns in the
# last segment; 9, 3, one segment of 255; 17, 5, one segment of 4; 22, 6, two segments, 85 columns in the last.
RUNS = [(6000, 777), (2100, 2303), (1300, 4100), (1000, 5461)]


@pytest.mark.parametrize("rows", ["padded", "dense", "offset"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D", RUNS)
def test_runs_of_four_segments(vl, guard, N, D, dtype, rows):
    segments = -(-D // 256)
    assert segments > 2 and N * -(-segments // 4) >= 148 * 5 * 8
    X = inputs(N, D, dtype, N + D, rows)
    q_ref, e_ref, xhat = definition(X)
    Q = guard.mat(N, D, torch.uint8).view(torch.int8)
    E = guard.mat(N, -(-D // BLOCK), torch.uint8)
    vl.velora_checkpoint_store(X, Q, E)
    assert np.array_equal(Q.cpu().numpy(), q_ref)
    assert np.array_equal(E.cpu().numpy(), e_ref)
    back = guard.mat(N, D, dtype, ld={"padded": None, "dense": D, "offset": D + 1 + D % 2}[rows])
    vl.velora_checkpoint_load(Q, E, back)
    equal_values(back, xhat)
