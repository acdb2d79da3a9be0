"""Rows in 8 bits: dynb_store8, dynb_load8 and the layer norm's gradients from them.

The format is fp32 arithmetic, step by step, so that the host's, which rounds the same way, has to give the same bits; the bound of an element's error
(half a scale) is checked beside it in 64 bits."""
import pytest
import torch

from tests.operator_util import U16, U32, gaps_untouched, stored, strided, within

pytestmark = pytest.mark.gpu
BF, F8 = torch.bfloat16, torch.float64


@pytest.fixture(scope="module")
def dyn():
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as d
    return d


def blocks(x):
    """[..., d] -> [..., blocks, 32], zeros behind the end"""
    d = x.shape[-1]
    return torch.nn.functional.pad(x, (0, -d % 32)).unflatten(-1, (-1, 32))


def to_eight(x):
    """The format, on the host in fp32: (q, scale)."""
    b = blocks(x.float())
    a = b.abs().amax(-1)
    fine = torch.isfinite(a)
    up = ((torch.where(fine, a, 0.0) / torch.full_like(a, 127.0)).view(torch.int32) + 0xffff) & -0x10000
    s = up.view(torch.float32).clamp(min=2.0 ** -126)
    q = torch.where(fine[..., None], torch.round(b * (torch.ones_like(s) / s)[..., None]), 0.0)
    return q.to(torch.int8).flatten(-2)[..., :x.shape[-1]], torch.where(fine, s, float("nan")).to(BF)


def values(q, scale):
    """What they stand for, in 64 bits."""
    return (blocks(q.double()) * scale.double()[..., None]).flatten(-2)[..., :q.shape[-1]]


def normal(T, d, dtype, seed, channels=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g)
    if channels:
        x = x * torch.exp(torch.randn(d, generator=g))
    return x.to(dtype)


SIZES = [(1, 1), (1, 32), (3, 31), (5, 33), (2, 64), (7, 100), (37, 512), (65, 1000), (129, 777), (300, 96), (4097, 40), (9, 5000), (2, 20011)]


@pytest.mark.parametrize("T,d", SIZES)
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_there_and_back(dyn, T, d, dtype):
    x = normal(T, d, dtype, T * 31 + d)
    got = dyn.dynb_store8(x.cuda())
    q, scale = to_eight(x)
    assert torch.equal(got.scale.cpu().view(torch.int16), scale.view(torch.int16))
    assert torch.equal(got.q.cpu(), q)
    want = values(q, scale)
    half = scale.double().repeat_interleave(32, -1)[:, :d] / 2
    assert bool(((want - x.double()).abs() <= half * (1 + 2.0 ** -15)).all())              # x * (1 / s) is rounded twice, 127 * 2^-23 of a step
    for to, code in ((BF, dyn.DYNB_BF16), (torch.float32, dyn.DYNB_F32)):
        assert torch.equal(dyn.dynb_load8(got, dtype=code).cpu(), want.to(to))


def test_ties_signs_and_the_smallest_and_largest_numbers(dyn):
    big = torch.finfo(torch.float32).max
    rows = [[0.0] * 40, [-0.0] * 40, [127.0] + [i + 0.5 for i in range(-20, 19)], [-127.0 * 2.0 ** -126] + [2.0 ** -127 * i for i in range(39)],
            [2.0 ** -149] * 40, [big] + [-big / i for i in range(1, 40)], [1.0] + [1e-30] * 39, [-3.0] * 40, [1e-38, 2e-39] * 20]
    x = torch.tensor(rows, dtype=torch.float32)
    got = dyn.dynb_store8(x.cuda())
    q, scale = to_eight(x)
    assert torch.equal(got.scale.cpu(), scale) and torch.equal(got.q.cpu(), q)
    back = dyn.dynb_load8(got, dtype=dyn.DYNB_F32).cpu()
    assert torch.equal(back, values(q, scale).float())      # (the largest numbers may come back as infinities)
    assert torch.equal(got.q.cpu()[2, 1:32].float(), torch.round(x[2, 1:32]))


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_a_block_with_what_is_no_number_is_nan_and_no_other(dyn, bad, dtype):
    x = normal(6, 100, dtype, 3)
    x[1, 0] = x[3, 63] = x[4, 99] = bad
    got = dyn.dynb_store8(x.cuda())
    q, scale = to_eight(x)
    assert torch.equal(got.q.cpu(), q)
    back = dyn.dynb_load8(got).cpu()
    lost = torch.zeros(6, 100, dtype=torch.bool)
    lost[1, :32] = lost[3, 32:64] = lost[4, 96:] = True
    assert torch.equal(torch.isnan(back), lost)
    assert torch.equal(back[~lost], values(q, scale)[~lost].to(BF))


@pytest.mark.parametrize("offset,gap", [(0, 8), (1, 3), (3, 0), (8, 16)])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_strides_and_addresses(dyn, offset, gap, dtype):
    for T, d in ((5, 100), (70, 64), (33, 257)):
        x = normal(T, d, dtype, d)
        n = (d + 31) // 32
        view, _ = strided(x, gap, dtype, offset)
        q, qb = strided(torch.zeros(T, d), gap, torch.int8, offset)
        s, sb = strided(torch.zeros(T, n), gap, BF, offset)
        kept = dyn.dynb_store8(view, out=dyn.Rows8(q, s))
        want = to_eight(x)
        assert torch.equal(q.cpu(), want[0]) and torch.equal(s.cpu(), want[1])
        back, bb = strided(torch.zeros(T, d), gap, dtype, offset)
        assert dyn.dynb_load8(kept, out=back) is back
        assert torch.equal(back.cpu(), values(*want).to(dtype))
        assert gaps_untouched(q, qb, offset) and gaps_untouched(s, sb, offset) and gaps_untouched(back, bb, offset)


def test_no_rows(dyn):
    got = dyn.dynb_store8(torch.empty(0, 40, device="cuda"))
    assert got.q.shape == (0, 40) and got.scale.shape == (0, 2) and dyn.dynb_load8(got).shape == (0, 40)


def test_rows_beyond_32_bits(dyn):
    """Offsets beyond 2^32 elements: a row far into a buffer, by its stride."""
    stride = (1 << 32) + 64
    buf = torch.empty(stride + 64, dtype=torch.int8, device="cuda")
    q = buf.as_strided((2, 64), (stride, 1))
    x = normal(2, 64, BF, 5)
    kept = dyn.dynb_store8(x.cuda(), out=dyn.Rows8(q, torch.empty(2, 2, dtype=BF, device="cuda")))
    want = to_eight(x)
    assert torch.equal(q.cpu(), want[0])
    assert torch.equal(dyn.dynb_load8(kept).cpu(), values(*want).to(BF))


NORMS = [(1, 1), (3, 40), (37, 512), (64, 777), (257, 1000), (130, 1024), (65, 2056), (40, 4096), (33, 5000), (20, 12288), (17, 16384), (9, 16400), (5, 20011)]


def norm_bounds(x, dy, gamma, mean, rstd):
    """Gradients in 64 bits and how far fp32 sums of d or T terms may be off."""
    d, T = x.shape[1], x.shape[0]
    h, g = (x - mean) * rstd, dy * gamma
    m1, m2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx = rstd * (g - m1 - h * m2)
    eh = 4 * U32 * ((x.abs() + mean.abs()) * rstd.abs())                                     # x - mean rounds once, rstd once more
    e2 = (d + 8) * 2 * U32 * (g * h).abs().mean(1, keepdim=True) + (g.abs() * eh).mean(1, keepdim=True)
    e1 = (d + 8) * 2 * U32 * g.abs().mean(1, keepdim=True)
    edx = rstd * (e1 + h.abs() * e2 + eh * m2.abs() + 8 * U32 * (g.abs() + m1.abs() + (h * m2).abs()))
    eg = (T + 8) * 2 * U32 * (dy * h).abs().sum(0) + (dy.abs() * eh).sum(0)
    return (dx, edx), ((dy * h).sum(0), eg), (dy.sum(0), (T + 8) * 2 * U32 * dy.abs().sum(0))


@pytest.mark.parametrize("T,d", NORMS)
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("gap", [0, 5])
def test_norm_gradients_from_eight_bits(dyn, T, d, dtype, gap):
    x, dy = normal(T, d, torch.float32, T + d) + 0.5, normal(T, d, dtype, T + d + 1, channels=False)
    g = torch.Generator().manual_seed(d)
    gamma = 1 + 0.2 * torch.randn(d, generator=g)
    q, scale = to_eight(x)
    _, mean, rstd = dyn.dynb_layer_norm(x.cuda(), gamma.cuda(), want_stats=True)
    qv, _ = strided(q, gap, torch.int8, gap)
    sv, _ = strided(scale, gap, BF, gap)
    dyv, _ = strided(dy, gap, dtype, gap)
    out, buf = strided(torch.zeros(T, d), gap, dtype, gap)
    dx, dgamma, dbeta = dyn.dynb_layer_norm_backward(dyv, dyn.Rows8(qv, sv), gamma.cuda(), mean, rstd, dx=out)
    assert dx is out and gaps_untouched(out, buf, gap)
    (rx, ex), (rg, eg), (rb, eb) = norm_bounds(values(q, scale), dy.double(), gamma.double(), mean.cpu().double()[:, None], rstd.cpu().double()[:, None])
    within(dx, rx, stored(rx, ex, dtype), "dx")
    within(dgamma, rg, eg + U32 * rg.abs(), "dgamma")
    within(dbeta, rb, eb + U32 * rb.abs(), "dbeta")
    again = dyn.dynb_layer_norm_backward(dyv, dyn.Rows8(qv, sv), gamma.cuda(), mean, rstd)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma) and torch.equal(again[2], dbeta)
    # exactly what the gradient of the restored rows is, where fp32 holds them
    if dtype == torch.float32 and gap == 0:
        plain = dyn.dynb_layer_norm_backward(dyv, dyn.dynb_load8(dyn.Rows8(qv, sv), dtype=dyn.DYNB_F32), gamma.cuda(), mean, rstd)
        within(dx, plain[0].double().cpu(), 2 * ex, "dx")


def test_norm_gradients_in_place_and_without_gamma(dyn):
    T, d = 50, 320
    x, dy = normal(T, d, torch.float32, 1), normal(T, d, BF, 2)
    kept = dyn.dynb_store8(x.cuda())
    _, mean, rstd = dyn.dynb_layer_norm(x.cuda(), want_stats=True)
    want = dyn.dynb_layer_norm_backward(dy.cuda(), kept, None, mean, rstd)
    buf = dy.cuda()
    got = dyn.dynb_layer_norm_backward(buf, kept, None, mean, rstd, dx=buf)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ones = dyn.dynb_layer_norm_backward(dy.cuda(), kept, torch.ones(d, device="cuda"), mean, rstd)
    assert all(torch.equal(a, b) for a, b in zip(ones, want))


def test_no_rows_have_no_gradients(dyn):
    kept = dyn.dynb_store8(torch.empty(0, 64, device="cuda"))
    none = torch.empty(0, device="cuda")
    _, dgamma, dbeta = dyn.dynb_layer_norm_backward(torch.empty(0, 64, device="cuda"), kept, None, none, none)
    assert not dgamma.any() and not dbeta.any()
