"""CPU-only checks of what velora_workspace_bytes answers for the flags of an operation."""
import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2405_17991_b200 import binding, build
    build.build()
    binding.lib()
    return binding


OLDER = ["OP_INIT_V", "OP_WEIGHT_GRAD_FACTORED", "OP_WEIGHT_GRAD_EXPLICIT", "OP_LINEAR_FORWARD", "OP_LINEAR_BACKWARD_FACTORED",
         "OP_LINEAR_BACKWARD_EXPLICIT", "OP_UPDATE_V", "OP_Z8_CALIBRATE"]


@pytest.mark.parametrize("name", OLDER)
def test_fp32_flag_belongs_to_three_operations(b, name):
    """The others have one size for both types: a flag that would mean nothing is refused."""
    size, op = b.lib().velora_workspace_bytes, getattr(b, name)
    assert size(op, 100, 64, 40, 8) > 0
    assert size(op | b.OP_F32, 100, 64, 40, 8) == 0
    assert size(op | b.OP_F32 | b.OP_ANY_ROWS, 100, 64, 40, 8) == 0


@pytest.mark.parametrize("name", ["OP_CHECKPOINT_WEIGHT_GRAD", "OP_HEAD_LOSS", "OP_HEAD_LOSS_BACKWARD"])
def test_fp32_flag_where_it_belongs(b, name):
    size, op = b.lib().velora_workspace_bytes, getattr(b, name)
    assert size(op | b.OP_F32, 300, 64, 40, 1) > 256
    assert size(op | 1024, 300, 64, 40, 1) == 0


@pytest.mark.parametrize("O", [40, 2056, 45])
def test_room_for_any_rows_of_the_checkpoint_gradient(b, O):
    """A bf16 dY may be a view on odd boundaries whatever its width: with the flag there is room for its packed copy, N rows of O rounded up to 8."""
    size, op, N, D = b.lib().velora_workspace_bytes, b.OP_CHECKPOINT_WEIGHT_GRAD, 300, 64
    assert size(op | b.OP_ANY_ROWS, N, D, O, 1) - size(op, N, D, O, 1) >= 2 * N * (-(-O // 8) * 8)
    assert size(op | b.OP_F32 | b.OP_ANY_ROWS, N, D, O, 1) == size(op | b.OP_F32, N, D, O, 1)
