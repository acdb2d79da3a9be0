"""Ways through the grouped products that ordinary sizes do not take, or not knowingly."""
import numpy as np
import pytest
import torch

from tests.operator_util import stored

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


def uneven(M, E, seed):
    """Loads from nothing to some hundred rows, and rows behind the last group."""
    r = np.random.Generator(np.random.Philox(key=[M + seed, E]))
    share = np.where((r.random(E) < 0.1) & (np.arange(E) > 0), 0.0, r.random(E) + 0.2)
    counts = np.bincount(r.choice(E, M - M // 50, p=share / share.sum()), minlength=E)
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


# 256 workgroups that stay look their tiles up 256 at a time: 8192 groups and more are never sorted, nor are more than 256 tiles a workgroup, which are looked up
# anew after every 256 (840000 rows: 164 of the workgroups have 257 and the others 256, and all have to go by the same numbering).  837600 rows and 8191 groups are
# the last that are sorted
@pytest.mark.parametrize("M,K,N,E", [(840_000, 64, 5120, 3), (900_000, 64, 5120, 3), (838_000, 64, 5120, 3), (837_600, 64, 5120, 3), (1_700_000, 64, 1280, 8192), (1_600_000, 128, 64, 8200),
                                     (1_600_000, 128, 64, 8191)])
def test_tiles_that_are_looked_up_as_they_come(dyn, M, K, N, E):
    g = torch.Generator("cuda").manual_seed(E)
    at = uneven(M, E, 1)
    off = torch.from_numpy(at).cuda()
    W = torch.randn(E, N, K, generator=g, device="cuda").mul_(K ** -0.5).to(BF)
    x = torch.randn((M + 1) // 2, K, generator=g, device="cuda").to(BF)
    perm = torch.randperm(M, generator=g, device="cuda").int()

    def check(got, rows_of, relu):
        """Every group's rows, 32768 at a time, against a product of its own."""
        assert torch.isfinite(got).all() and not got[at[-1]:].any()
        for e in range(E):
            w = W[e].double().t().contiguous() if at[e + 1] > at[e] else None
            for lo in range(at[e], at[e + 1], 32768):
                rows, hi = rows_of(lo, min(at[e + 1], lo + 32768)), min(at[e + 1], lo + 32768)
                ref = (rows @ w).clamp(min=0) if relu else rows @ w
                wrong.append(((got[lo:hi].double() - ref).abs() > stored(ref, K * 2.0 ** -23 * (rows.abs() @ w.abs()), BF)).any())

    wrong = []
    out = torch.full((M, N), float("nan"), dtype=BF, device="cuda")
    dyn.moe_product(x, W, off, perm=perm, k=2, relu=True, out=out)
    check(out, lambda lo, hi: x[perm[lo:hi].long() // 2].double(), True)
    del out
    # the input's gradient of the turned layer: N channels into K features
    V = W.transpose(1, 2).contiguous()                           # [E][K][N]
    dout = torch.randn(M, K, generator=g, device="cuda").to(BF)
    din = torch.full((M, N), float("nan"), dtype=BF, device="cuda")
    dyn.moe_product_grad_input(dout, V, off, out=din)
    check(din, lambda lo, hi: dout[lo:hi].double(), False)
    assert int(torch.stack(wrong).sum()) == 0


def agrees(got, ref, err):
    """Results stored in bfloat16, on the device: within `err` of ref before they were rounded (operator_util.stored)."""
    return bool(((got.double() - ref).abs() <= stored(ref, err, got.dtype)).all())


@pytest.mark.parametrize("M,K,N,E", [(300, 64, 72, 2047), (300, 64, 72, 2048), (300, 64, 64, 5000), (9000, 40, 64, 5000), (300, 63, 65, 5000), (700, 32, 16, 70000), (700, 31, 17, 70000), (90000, 16, 24, 20000)])
def test_groups_by_the_thousand(dyn, M, K, N, E):
    """Rows find their groups in several steps of a search, and fewer rows than groups."""
    g = torch.Generator("cuda").manual_seed(E + K)
    at = uneven(M, E, 2)
    off = torch.from_numpy(at).cuda()
    live, used = int(at[-1]), torch.from_numpy(np.searchsorted(at, np.arange(M), side="right") - 1).cuda()
    W = torch.randn(E, N, K, generator=g, device="cuda").mul_(K ** -0.5).to(BF)
    x, dout = torch.randn(M, K, generator=g, device="cuda").to(BF), torch.randn(M, N, generator=g, device="cuda").to(BF)
    out = dyn.moe_product(x, W, off, out=torch.full((M, N), float("nan"), dtype=BF, device="cuda"))
    din = dyn.moe_product_grad_input(dout, W, off, out=torch.full((M, K), float("nan"), dtype=BF, device="cuda"))
    assert not out[live:].any() and not din[live:].any()
    for lo in range(0, live, 3000):
        hi = min(live, lo + 3000)
        w, xs, ds = W[used[lo:hi]].double(), x[lo:hi].double(), dout[lo:hi].double()
        assert agrees(out[lo:hi], (w * xs[:, None, :]).sum(2), K * 2.0 ** -23 * (w * xs[:, None, :]).abs().sum(2)), (lo, hi)
        assert agrees(din[lo:hi], (w * ds[:, :, None]).sum(1), N * 2.0 ** -23 * (w * ds[:, :, None]).abs().sum(1)), (lo, hi)
    ref, mag = torch.zeros(E, N * K, dtype=torch.float64, device="cuda"), torch.zeros(E, N * K, dtype=torch.float64, device="cuda")
    for lo in range(0, live, 3000):
        hi = min(live, lo + 3000)
        outer = (dout[lo:hi].double()[:, :, None] * x[lo:hi].double()[:, None, :]).flatten(1)
        ref.index_add_(0, used[lo:hi], outer)
        mag.index_add_(0, used[lo:hi], outer.abs())
    longest = int(np.diff(at).max())
    dW = dyn.moe_product_grad_weight(dout, x, off, dW=torch.full((E, N, K), float("nan"), device="cuda"))
    assert agrees(dW.view(E, -1), ref, longest * 2.0 ** -23 * mag)
