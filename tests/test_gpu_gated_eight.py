"""The pair that moe_gated keeps in 8 bits is the format's, step by step in fp32 (include/dynbatch.h: dynb_rows8): where gate and up are known to the last bit, so are the scales and
the elements, and dynb_store8 of the same numbers gives the same bits.

Two channels alone have weights: gate is x[r, 0] Wg[f, 0] and up x[r, 1] Wu[f, 1], products of 8 by 8 bits of significand, and every other term of their sums is 0: exact in fp32
in any order.  Weights are halves, (n + 1/2), and 127, so that x / s lies on the middle between two whole numbers nearly everywhere: a product that is not rounded before it is rounded
to a whole number goes to the other neighbour in two of five such places."""
import pytest
import torch

from tests.test_gpu_gated import BF, code, dyn  # noqa: F401
from tests.test_gpu_rows8 import to_eight
from tests.tile_kinds import kind_of

pytestmark = pytest.mark.gpu


def known(M, K, h, E, seed):
    """x, W of moe_gated and the gate and up that they give, [M, 2, h] in fp32"""
    g = torch.Generator().manual_seed(seed)
    x, W = torch.zeros(M, K), torch.zeros(E, 2, h, K)
    for s in range(2):
        halves = torch.randint(0, 127, (E, h), generator=g) + 0.5
        halves[:, torch.arange(h) % 32 == min(5, h - 1)] = 127.0             # the largest of every block, also of a short one behind
        halves[:, -1] = 127.0
        W[:, s, :, s] = halves * (torch.randint(0, 2, (E, h), generator=g) * 2 - 1)
        x[:, s] = torch.randint(128, 256, (M,), generator=g) * 2.0 ** torch.randint(-20, 10, (M,), generator=g)
        x[:, s] *= torch.randint(0, 2, (M,), generator=g) * 2 - 1
    off = torch.linspace(0, M - M // 9, E + 1).int()
    expert = torch.searchsorted(off[1:].contiguous(), torch.arange(M).int(), right=True)
    pre = torch.zeros(M, 2, h)
    for s in range(2):
        rows = expert < E
        pre[rows, s] = x[rows, s, None] * W[expert[rows], s, :, s]
    return x.to(BF), W.to(BF), off, pre


# rows, channels, hidden features, experts, the tile that they go to, and whether rows are on borders
@pytest.mark.parametrize("M,K,h,E,kind,border", [
    (5, 64, 96, 2, "few", True), (70, 128, 200, 3, "few", True), (70, 130, 203, 3, "few", False), (3, 5, 31, 1, "few", False), (2000, 72, 1040, 4, "mid", True),
    (2000, 72, 1032, 4, "mid", True), (2000, 75, 1001, 4, "mid", False), (40000, 520, 2064, 12, "big", True), (40000, 520, 2056, 12, "big", True)])
def test_the_pair_is_the_formats(dyn, M, K, h, E, kind, border):  # noqa: F811
    assert kind_of(M, E, 2 * h, K) == kind and border == (K % 8 == 0 and h % 8 == 0)
    x, W, off, pre = known(M, K, h, E, M + h)
    kept = dyn.Rows8(torch.full((M, 2, h), 77, dtype=torch.int8, device="cuda"), torch.full((M, 2, (h + 31) // 32), 7.0, dtype=BF, device="cuda"))
    exact = torch.empty(M, 2, h, dtype=BF, device="cuda")
    for gate in ("silu", "gelu"):
        dyn.moe_gated(x.cuda(), W.cuda(), off.cuda(), gate=code(dyn, gate), pre=kept)
        part = slice(0, M) if M < 5000 else torch.randint(0, M, (3000,), generator=torch.Generator().manual_seed(1))
        q, s = to_eight(pre[part])
        assert torch.equal(kept.scale.cpu()[part].view(torch.int16), s.view(torch.int16))
        assert torch.equal(kept.q.cpu()[part], q)
        for i in range(2):
            again = dyn.dynb_store8(pre[:, i].contiguous().cuda())
            assert torch.equal(again.q, kept.q[:, i]) and torch.equal(again.scale, kept.scale[:, i])
    dyn.moe_gated(x.cuda(), W.cuda(), off.cuda(), pre=exact)
    assert torch.equal(exact.cpu(), pre.to(BF))


@pytest.mark.parametrize("h", [64, 100])
def test_the_smallest_and_largest_blocks(dyn, h):  # noqa: F811
    """Blocks whose scale is held at 2^-126, blocks of zeros, and blocks next to the largest number of fp32"""
    M, K = 40, 8
    g = torch.Generator().manual_seed(h)
    x, W = torch.zeros(M, K), torch.zeros(1, 2, h, K)
    power = torch.arange(M) - 20
    weights = lambda: (torch.randint(64, 256, (h,), generator=g) * (torch.randint(0, 2, (h,), generator=g) * 2 - 1)).float()
    x[:, 0], x[:, 1] = 2.0 ** (power - 60.0), 2.0 ** (110.0 + power.clamp(max=10))
    W[0, 0, :, 0], W[0, 1, :, 1] = weights() * 2.0 ** -60, weights()
    x[7], x[9] = 0.0, -0.0
    pre = torch.stack([x[:, :1] * W[0, 0, :, 0], x[:, 1:2] * W[0, 1, :, 1]], 1)
    assert torch.isfinite(pre).all() and float(pre.max()) > 2.0 ** 127
    keep = (pre[:, 0].abs() >= 2.0 ** -126).all(1) | (pre[:, 0] == 0).all(1)  # (what matrix instructions make of smaller products is not the format's)
    kept = dyn.Rows8(torch.empty(M, 2, h, dtype=torch.int8, device="cuda"), torch.empty(M, 2, (h + 31) // 32, dtype=BF, device="cuda"))
    dyn.moe_gated(x.to(BF).cuda(), W.to(BF).cuda(), torch.tensor([0, M], dtype=torch.int32, device="cuda"), pre=kept)
    q, s = to_eight(pre)
    assert bool((s[keep, 0] == 2.0 ** -126).all(1).sum() > 4)                # (zeros are two of them)
    assert torch.equal(kept.q.cpu()[:, 1], q[:, 1]) and torch.equal(kept.scale.cpu()[:, 1], s[:, 1])
    assert torch.equal(kept.q.cpu()[keep, 0], q[keep, 0]) and torch.equal(kept.scale.cpu()[keep, 0], s[keep, 0])
