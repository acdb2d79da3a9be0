"""What the binding of the gated layer and of the rows in 8 bits refuses: tensors that are not what their documentation says, which the C side cannot see."""
import pytest
import torch

from tests.test_gpu_gated import BF, dyn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(4, 2), (4, 1), (5,), (3,)])
def test_offsets_are_one_row_of_borders(dyn, shape):  # noqa: F811
    x, W, off = torch.ones(6, 16, dtype=BF, device="cuda"), torch.ones(3, 2, 8, 16, dtype=BF, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")
    with pytest.raises(AssertionError):
        dyn.moe_gated(x, W, off)
    with pytest.raises(AssertionError):
        dyn.moe_gated_grad(x, torch.ones(3, 16, 8, dtype=BF, device="cuda"), off, torch.ones(6, 2, 8, dtype=BF, device="cuda"))


@pytest.mark.parametrize("dtype", [2, -1])
def test_rows_are_restored_in_bfloat16_or_float32(dyn, dtype):  # noqa: F811
    with pytest.raises(AssertionError):
        dyn.dynb_load8(dyn.dynb_store8(torch.ones(3, 40, device="cuda")), dtype=dtype)
