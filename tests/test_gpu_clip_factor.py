"""dynb_clip_gradients where max_norm / norm is below fp32's normal range (2^-126): the gradients are still g * max_norm / norm, off by
their own rounding and by the norm's to fp32."""
import pytest
import torch

from tests.operator_util import U16, U32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dyn():
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as d
    return d


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size,max_norm", [(1e37, 1e-3), (1e37, 1e-6), (2e36, 0.9e-1), (1e37, 1.0)])
def test_factors_below_the_normal_range(dyn, dtype, size, max_norm):
    g = torch.Generator().manual_seed(5)
    grads = [(torch.rand(n, generator=g) + 0.5).mul(size).to(dtype).cuda() for n in (400, 7, 33)]
    kept = [t.double().cpu() for t in grads]
    norm = float(torch.cat(kept).square().sum().sqrt())
    assert norm < 3.4e38 and max_norm / norm < 2.0 ** -120
    assert abs(float(dyn.dynb_clip_gradients(grads, max_norm)) - norm) <= 4 * U32 * norm
    for t, k in zip(grads, kept):
        want = k * (float(torch.tensor(max_norm)) / norm)
        assert ((t.double().cpu() - want).abs() <= ((U16 if dtype == torch.bfloat16 else U32) + 8 * U32) * want).all()
