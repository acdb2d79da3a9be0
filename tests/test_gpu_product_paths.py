"""Ways through the grouped products that ordinary sizes do not take, or not knowingly."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def dyn():
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as d
    return d


def offsets_of(M, E, seed, power=3.0):
    """Skewed loads, every third group empty where there are several."""
    r = np.random.Generator(np.random.Philox(key=[M, seed]))
    share = r.random(E) ** power
    if E > 2:
        share[::3] = 0
    return torch.from_numpy(np.concatenate([[0], np.cumsum(np.bincount(r.choice(E, M, p=share / share.sum()), minlength=E))]).astype(np.int32)).cuda()


@pytest.mark.parametrize("M,K,N,E", [(8200, 2048, 2048, 1), (16384, 2048, 1928, 20), (65536, 256, 512, 300), (4500, 256, 264, 1), (3001, 320, 192, 40), (4500, 255, 257, 3), (40, 64, 64, 9)])
@pytest.mark.parametrize("gathered", [False, True])
def test_a_bfloat16_gradient_is_the_fp32_gradient_rounded_once(dyn, M, K, N, E, gathered):
    """Both types add up the same products in the same order, whole groups and those that borders cut alike."""
    g = torch.Generator("cuda").manual_seed(M + K)
    off = offsets_of(M, E, 1)
    x, dout = torch.randn(M, K, generator=g, device="cuda").to(BF), torch.randn(M, N, generator=g, device="cuda").to(BF)
    how = dict(perm=torch.randperm(2 * M, generator=g, device="cuda")[:M].int(), k=2) if gathered else {}
    wide = dyn.moe_product_grad_weight(dout, x, off, dW=torch.full((E, N, K), float("nan"), device="cuda"), **how)
    narrow = dyn.moe_product_grad_weight(dout, x, off, dW=torch.full((E, N, K), float("nan"), dtype=BF, device="cuda"), **how)
    assert torch.isfinite(wide).all()
    assert torch.equal(narrow, wide.to(BF))
