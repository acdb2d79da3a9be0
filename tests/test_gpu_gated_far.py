"""Gated layers with rows that lie further apart than 32 bits of elements reach, and with more tiles and groups than a workgroup's list and LDS hold."""
import pytest
import torch

from tests.operator_util import stored, within
from tests.test_gpu_gated import BF, bf, dyn, forward_ref, grad_ref, layout  # noqa: F401

pytestmark = pytest.mark.gpu


def apart(rows, stride, like):
    """Rows of `like`'s shape, `stride` elements apart"""
    whole = torch.empty((rows - 1) * stride + like[0].numel(), dtype=like.dtype, device="cuda")
    return whole.as_strided(like.shape, (stride,) + tuple(like.stride()[1:]))


# Equal sums in equal kernels are equal bits: what lies next to each other is the reference.  33 rows of scales 2^27 apart end at 2^32 elements, where 32 bits do;
# 2^27 + 2^20 apart they pass it, and the layer for any size runs, as it does for the reference where one more element between rows of out takes them off their borders.
@pytest.mark.parametrize("M", [33, 40])
@pytest.mark.parametrize("scale_stride", [1 << 27, (1 << 27) + (1 << 20), (1 << 28) + 1])
def test_rows_kept_far_apart(dyn, M, scale_stride):  # noqa: F811
    K, h = 64, 96
    g, _, off = layout(M, 1, "last", M)
    x, W = bf(g, M, K).to(BF).cuda(), bf(g, 1, 2, h, K, std=K ** -0.5).to(BF).cuda()
    new = lambda: dyn.Rows8(torch.empty(M, 2, h, dtype=torch.int8, device="cuda"), torch.empty(M, 2, 3, dtype=BF, device="cuda"))
    near, far = new(), new()
    far = dyn.Rows8(apart(M, 1 << 28, far.q), apart(M, scale_stride, far.scale))
    on_border = scale_stride <= 1 << 27
    out = torch.empty(M, h + 1, dtype=BF, device="cuda")[:, :h]
    want = dyn.moe_gated(x, W, off, out=None if on_border else out, pre=near)
    got = dyn.moe_gated(x, W, off, pre=far)
    assert torch.equal(got, want) and torch.equal(far.q, near.q) and torch.equal(far.scale, near.scale)
    W2, dout = bf(g, 1, K, h, std=K ** -0.5).to(BF).cuda(), bf(g, M, K).to(BF).cuda()
    hid = torch.empty(M, h + 1, dtype=BF, device="cuda")[:, :h]
    want = dyn.moe_gated_grad(dout, W2, off, near, hidden=None if on_border else hid)
    got = dyn.moe_gated_grad(dout, W2, off, far)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("stride", [1 << 27, (1 << 27) + 1])
def test_results_far_apart(dyn, stride):  # noqa: F811
    M, K, h = 40, 64, 96
    g, _, off = layout(M, 1, "last", M)
    x, W = bf(g, M, K).to(BF).cuda(), bf(g, 1, 2, h, K, std=K ** -0.5).to(BF).cuda()
    new = lambda *s: torch.empty(*s, dtype=BF, device="cuda")
    gap = stride % 8
    pre = new(M, 2 * h + gap)[:, :2 * h].unflatten(1, (2, h))
    want = dyn.moe_gated(x, W, off, pre=pre)
    out, kept = apart(M, stride, new(M, h)), apart(M, stride, new(M, 2, h))
    dyn.moe_gated(x, W, off, out=out, pre=kept)
    assert torch.equal(out, want) and torch.equal(kept, pre)
    W2, dout = bf(g, 1, K, h, std=K ** -0.5).to(BF).cuda(), bf(g, M, K).to(BF).cuda()
    want, hid = dyn.moe_gated_grad(dout, W2, off, pre)
    dpre, hidden = apart(M, stride, new(M, 2, h)), out
    dyn.moe_gated_grad(dout, W2, off, kept, dpre=dpre, hidden=hidden)
    assert torch.equal(dpre, want) and torch.equal(hidden, hid)


# 64 groups, more tiles of 256 x 256 than 256 workgroups list at once; 8192 groups, whose counts LDS does not hold; both.  Checked at the rows of a few groups, first and last among them.
@pytest.mark.parametrize("M,h,E", [(1 << 19, 4096, 64), (192 * 8192 + 77, 256, 8192), (192 * 8192 + 77, 2048, 8192)])
def test_many_tiles(dyn, M, h, E):  # noqa: F811
    K, N = 64, 64
    gen = torch.Generator(device="cuda").manual_seed(M + h)
    share = torch.rand(E, generator=torch.Generator().manual_seed(E)) + 0.05
    share[1] = 0                                              # a group without rows
    rows = torch.bincount(torch.multinomial(share, M, replacement=True, generator=torch.Generator().manual_seed(h)), minlength=E)
    off = torch.cat([torch.zeros(1, dtype=torch.long), rows.cumsum(0)])
    off_d = off.int().cuda()
    x = torch.randn(M, K, generator=gen, device="cuda").to(BF)
    W = (torch.randn(E, 2, h, K, generator=gen, device="cuda") * 0.125).to(BF)
    out = dyn.moe_gated(x, W, off_d)
    pre = torch.empty(M, 2, h, dtype=BF, device="cuda")
    assert torch.equal(dyn.moe_gated(x, W, off_d, pre=pre), out)
    dout = torch.randn(M, N, generator=gen, device="cuda").to(BF)
    W2 = (torch.randn(E, N, h, generator=gen, device="cuda") * 0.125).to(BF)
    dpre, hidden = dyn.moe_gated_grad(dout, W2, off_d, pre)
    for e in (0, 1, 2, E // 2, E - 1):
        a, b = int(off[e]), int(off[e + 1])
        few = slice(a, min(b, a + 300)) if e % 2 == 0 else slice(max(a, b - 300), b)
        n = few.stop - few.start
        if n == 0:
            continue
        of = lambda t: t[few].cpu().double()
        kept, err, ref, bound = forward_ref(of(x), W[e:e + 1].cpu().double(), [0, n], of(x), "silu")
        within(out[few], ref, stored(ref, bound, BF), f"out of group {e}")
        within(pre[few], kept, stored(kept, err, BF), f"kept of group {e}")
        (dg, bg), (du, bu), (hid, bh) = grad_ref(of(dout), W2[e:e + 1].cpu().double(), [0, n], of(pre), "silu")
        for what, got, ref, bound in (("dgate", dpre[few, 0], dg, bg), ("dup", dpre[few, 1], du, bu), ("hidden", hidden[few], hid, bh)):
            within(got, ref, stored(ref, bound, BF), f"{what} of group {e}")
