"""moe_gated and moe_gated_grad against the formulas in 64 bits, expert by expert.

Bounds.  gate and up are sums of K products (tests/operator_util.py): off by dg, du.  sigma's argument p = g (a + b g^2) is rounded four times (4 U32 |p|, which
sigma passes on relative to itself), exp2's argument once more, exponential, sum and reciprocal to 2 U32 each, and sigma <= 1: 8 (1 + |p|) U32 in all.  |f'| <= 1.13.
The slope sigma + sigma (1 - sigma) w, w = c (a + 3 b c^2): both terms relative as above, and 1 - sigma to 2 U32 absolute.  The reciprocal
gives 0 for a sigma below 2^-126, the smallest normal number: f = g sigma is then off by up to |g| 2^-126 (at g = -88, 1.03e-36), the slope by (1 + 2 |w|) 2^-126."""
import math

import numpy as np
import pytest
import torch

from tests.operator_util import U32, gaps_untouched, stored, strided, within
from tests.test_gpu_product import SHAPES, counts_of
from tests.test_gpu_rows8 import blocks, to_eight, values

pytestmark = pytest.mark.gpu
BF, F8 = torch.bfloat16, torch.float64
TINY = 2.0 ** -126


@pytest.fixture(scope="module")
def dyn():
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as d
    return d


def bf(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, dtype=F8) * std).to(BF).double()


def dev(t, dtype=BF):
    return t.to(dtype).cuda()


GATES = {"silu": (1.0, 0.0), "gelu": (2 * math.sqrt(2 / math.pi), 2 * math.sqrt(2 / math.pi) * 0.044715)}


def code(dyn, gate):
    return dyn.MOE_GATE_SILU if gate == "silu" else dyn.MOE_GATE_GELU


def gate_of(gate, g):
    """f, f', and bounds of their errors in fp32 for an exact g"""
    a, b = GATES[gate]
    p, w = g * (a + b * g * g), g * (a + 3 * b * g * g)
    s, away = torch.sigmoid(p), torch.sigmoid(-p)
    rel = 8 * (1 + p.abs()) * U32
    f, slope = g * s, s + s * away * w
    return f, slope, (rel + 2 * U32) * f.abs() + g.abs() * TINY, rel * (s + 2 * s * away * w.abs()) + 4 * U32 * s * w.abs() + (1 + 2 * w.abs()) * TINY


def forward_ref(x, W, off, rows, gate):
    """gate and up [M,2,h] and the bound of their errors, out and its"""
    M, h = len(rows), W.shape[2]
    pre, err = torch.zeros(M, 2, h, dtype=F8), torch.zeros(M, 2, h, dtype=F8)
    for e in range(W.shape[0]):
        a, b = int(off[e]), int(off[e + 1])
        for s in range(2):
            pre[a:b, s] = rows[a:b] @ W[e, s].t()
            err[a:b, s] = rows.shape[1] * 2 * U32 * (rows[a:b].abs() @ W[e, s].abs().t())
    f, _, ef, _ = gate_of(gate, pre[:, 0])
    out = f * pre[:, 1]
    bound = (1.13 * err[:, 0] + ef) * (pre[:, 1].abs() + err[:, 1]) + f.abs() * err[:, 1] + 2 * U32 * out.abs()
    return pre, err, out, bound


def grad_ref(dout, W, off, pre, gate):
    """dgate, dup, hidden and their bounds"""
    M, h = pre.shape[0], pre.shape[2]
    dact, err = torch.zeros(M, h, dtype=F8), torch.zeros(M, h, dtype=F8)
    live = torch.zeros(M, 1, dtype=F8)
    for e in range(W.shape[0]):
        a, b = int(off[e]), int(off[e + 1])
        dact[a:b] = dout[a:b] @ W[e]
        err[a:b] = dout.shape[1] * 2 * U32 * (dout[a:b].abs() @ W[e].abs())
        live[a:b] = 1
    f, slope, ef, es = gate_of(gate, pre[:, 0])
    u = pre[:, 1]
    dg, du, hid = dact * u * slope, dact * f, live * f * u
    bg = u.abs() * (err * (slope.abs() + es) + dact.abs() * es) + 4 * U32 * dg.abs()
    bu = err * (f.abs() + ef) + dact.abs() * ef + 4 * U32 * du.abs()
    return (dg, bg), (du, bu), (hid, live * (ef * u.abs() + 4 * U32 * hid.abs()))


def layout(M, E, loads, seed):
    g = torch.Generator().manual_seed(seed)
    off = np.concatenate([[0], np.cumsum(counts_of(loads, M, E, g))]).astype(np.int32)
    return g, off, torch.from_numpy(off).cuda()


def check_eight(kept, pre, err):
    """Kept pairs in 8 bits: the scale that the largest number of a block may have, elements within half of it"""
    s, q = kept.scale.cpu(), kept.q.cpu()
    largest, slack = blocks(pre.abs()).amax(-1), blocks(err).amax(-1)
    up = lambda v: ((v.clamp(min=0).float() / 127).view(torch.int32) + 0xffff).bitwise_and(-0x10000).view(torch.float32).clamp(min=2.0 ** -126)
    room = 1 + 4 * U32
    assert bool((s.float() >= up((largest - slack) / room)).all()) and bool((s.float() <= up((largest + slack) * room)).all())
    half = s.double().repeat_interleave(32, -1)[..., :pre.shape[-1]] / 2
    assert bool(((values(q, s) - pre).abs() <= half * (1 + 2.0 ** -15) + err).all())


@pytest.mark.parametrize("M,K,h,E,loads", SHAPES)
@pytest.mark.parametrize("gate,gathered", [("silu", False), ("gelu", True), ("silu", True)])
def test_forward(dyn, M, K, h, E, loads, gate, gathered):
    g, off, off_d = layout(M, E, loads, M * 7 + K)
    k = 3 if gathered else 1
    n_rows = (M + k - 1) // k if gathered else M
    x, W = bf(g, n_rows, K), bf(g, E, 2, h, K, std=K ** -0.5)
    perm = torch.randperm(M, generator=g).int() if gathered else None
    rows = x[perm.long() // k] if gathered else x
    pre, err, ref, bound = forward_ref(x, W, off, rows, gate)
    n = (h + 31) // 32
    kept8 = dyn.Rows8(torch.full((M, 2, h), 77, dtype=torch.int8, device="cuda"), torch.full((M, 2, n), 7.0, dtype=BF, device="cuda"))
    kept16 = torch.full((M, 2, h), float("nan"), dtype=BF, device="cuda")
    got = {}
    for what, keep in (("nothing", None), ("bf16", kept16), ("eight", kept8)):
        out = torch.full((M, h), float("nan"), dtype=BF, device="cuda")
        assert dyn.moe_gated(dev(x), dev(W), off_d, perm=perm.cuda() if gathered else None, k=k, gate=code(dyn, gate), out=out, pre=keep) is out
        within(out, ref, stored(ref, bound, BF), what)
        got[what] = out
    within(kept16, pre, stored(pre, err, BF), "kept")
    check_eight(kept8, pre, err)
    again = dyn.moe_gated(dev(x), dev(W), off_d, perm=perm.cuda() if gathered else None, k=k, gate=code(dyn, gate))
    assert torch.equal(again, got["nothing"])


@pytest.mark.parametrize("M,N,h,E,loads", SHAPES)
@pytest.mark.parametrize("gate,eight,want_hidden", [("silu", False, True), ("gelu", True, True), ("silu", True, False)])
def test_grad(dyn, M, N, h, E, loads, gate, eight, want_hidden):
    g, off, off_d = layout(M, E, loads, M * 11 + N)
    dout, W, pre = bf(g, M, N), bf(g, E, N, h, std=N ** -0.5), bf(g, M, 2, h, std=2.0)
    kept = dev(pre)
    if eight:
        q, s = to_eight(pre)
        pre, kept = values(q, s), dyn.Rows8(q.cuda(), s.cuda())
    (dg, bg), (du, bu), (hid, bh) = grad_ref(dout, W, off, pre, gate)
    dpre = torch.full((M, 2, h), float("nan"), dtype=BF, device="cuda")
    hidden = torch.full((M, h), float("nan"), dtype=BF, device="cuda") if want_hidden else None
    got = dyn.moe_gated_grad(dev(dout), dev(W), off_d, kept, gate=code(dyn, gate), dpre=dpre, hidden=hidden, want_hidden=want_hidden)
    assert (got[0] if want_hidden else got) is dpre
    within(dpre[:, 0], dg, stored(dg, bg, BF), "gate")
    within(dpre[:, 1], du, stored(du, bu, BF), "up")
    if want_hidden:
        within(hidden, hid, stored(hid, bh, BF), "hidden")
    again = dyn.moe_gated_grad(dev(dout), dev(W), off_d, kept, gate=code(dyn, gate))
    assert torch.equal(again[0], dpre) and (not want_hidden or torch.equal(again[1], hidden))


@pytest.mark.parametrize("gap,offset", [(8, 0), (16, 8), (5, 1), (0, 3)])
@pytest.mark.parametrize("M,K,h,E", [(70, 64, 96, 4), (300, 136, 200, 3), (33, 40, 31, 2)])
def test_strides_and_addresses(dyn, M, K, h, E, gap, offset):
    g, off, off_d = layout(M, E, "tail", M + gap)
    x, W, n = bf(g, M, K), bf(g, E, 2, h, K, std=K ** -0.5), (h + 31) // 32
    pre, err, ref, bound = forward_ref(x, W, off, x, "silu")
    xv, _ = strided(x, gap, BF, offset)
    out, ob = strided(torch.zeros(M, h), gap, BF, offset)
    p16, b16 = strided(torch.zeros(M, 2 * h), gap, BF, offset)
    q, qb = strided(torch.zeros(M, 2 * h), gap, torch.int8, offset)
    s, sb = strided(torch.zeros(M, 2 * n), gap, BF, offset)
    kept16, kept8 = p16.unflatten(1, (2, h)), dyn.Rows8(q.unflatten(1, (2, h)), s.unflatten(1, (2, n)))
    for keep in (kept16, kept8):
        out.zero_()
        dyn.moe_gated(xv, dev(W), off_d, out=out, pre=keep)
        within(out, ref, stored(ref, bound, BF))
    within(kept16, pre, stored(pre, err, BF))
    check_eight(kept8, pre, err)
    for view, buf in ((out, ob), (p16, b16), (q, qb), (s, sb)):
        assert gaps_untouched(view, buf, offset)
    # backward, from either
    N = K
    dout, W2 = bf(g, M, N), bf(g, E, N, h, std=N ** -0.5)
    dv, _ = strided(dout, gap, BF, offset)
    for keep, stand in ((kept16, kept16.double().cpu()), (kept8, values(kept8.q.cpu(), kept8.scale.cpu()))):
        (dg, bg), (du, bu), (hid, bh) = grad_ref(dout, W2, off, stand, "silu")
        d16, db = strided(torch.zeros(M, 2 * h), gap, BF, offset)
        hv, hb = strided(torch.zeros(M, h), gap, BF, offset)
        dyn.moe_gated_grad(dv, dev(W2), off_d, keep, dpre=d16.unflatten(1, (2, h)), hidden=hv)
        within(d16[:, :h], dg, stored(dg, bg, BF))
        within(d16[:, h:], du, stored(du, bu, BF))
        within(hv, hid, stored(hid, bh, BF))
        assert gaps_untouched(d16, db, offset) and gaps_untouched(hv, hb, offset)


def test_far_values_of_the_gate(dyn):
    """One channel and features with one weight each: the gate takes any number.  Infinities and NaN as the formula has them."""
    g = torch.cat([torch.linspace(-120, 120, 481), torch.tensor([1e-30, -1e-30, 1e4, -1e4, 3e18, -3e18, 1e30, -1e30, 3e38, -3e38, float("inf"), float("nan"), 0.0, -0.0])]).to(BF)
    M = len(g)
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    W = torch.ones(1, 2, 8, 8, dtype=BF)
    W[0, :, :, 1:] = 0
    W[0, 1] = 0
    W[0, 1, :, 1] = 1                                        # up: the second channel, which is 1
    x = torch.zeros(M, 8, dtype=BF)
    x[:, 0], x[:, 1] = g, 1.0
    gd = g.double()
    finite = torch.isfinite(gd)
    for gate in GATES:
        kept = torch.empty(M, 2, 8, dtype=BF, device="cuda")
        out = dyn.moe_gated(x.cuda(), W.cuda(), off, gate=code(dyn, gate), pre=kept)[:, 0].cpu().double()
        f, slope, ef, es = gate_of(gate, gd.clamp(-1e4, 1e4))    # (sigma is 0 or 1 from there on)
        f = torch.where(gd.abs() > 1e4, gd * torch.sigmoid(gd), f)
        assert math.isnan(out[-4]) and math.isnan(out[-3])       # (an infinity times up's zero weight is none)
        within(out[finite], f[finite], stored(f, ef * (1 + gd.abs() / 1e4), BF)[finite])
        # backward: dact 1, up 1
        ones, W2 = torch.zeros(M, 8, dtype=BF), torch.zeros(1, 8, 8, dtype=BF)
        ones[:, 0], W2[0, 0] = 1.0, 1.0
        pre = torch.ones(M, 2, 8, dtype=BF)
        pre[:, 0] = g[:, None]
        dpre, hidden = dyn.moe_gated_grad(ones.cuda(), W2.cuda(), off, pre.cuda(), gate=code(dyn, gate))
        within(dpre[:, 0, 0].cpu()[finite], slope[finite], stored(slope, es, BF)[finite])
        within(dpre[:, 1, 0].cpu()[finite], f[finite], stored(f, ef * (1 + gd.abs() / 1e4), BF)[finite])
        assert torch.equal(dpre[:, 1, 0][torch.isfinite(hidden[:, 0])], hidden[:, 0][torch.isfinite(hidden[:, 0])])
        assert float(dpre[-4, 0, 0]) == 1.0 and torch.isnan(dpre[-3]).all()


def test_what_no_group_has_is_zero_whatever_it_was(dyn):
    """Rows behind the last group: results are 0, also where what was kept there is no number; the rows of groups next to NaN rows keep theirs."""
    M, K, h, E = 150, 64, 64, 2
    g = torch.Generator().manual_seed(1)
    off = torch.tensor([0, 40, 90], dtype=torch.int32, device="cuda")
    x, W = dev(bf(g, M, K)), dev(bf(g, E, 2, h, K, std=0.1))
    x[90:] = float("nan")
    x[5] = float("nan")
    for n in (h, h - 1):
        Wn = W[:, :, :n].contiguous()
        kept = dyn.Rows8(torch.empty(M, 2, n, dtype=torch.int8, device="cuda"), torch.empty(M, 2, (n + 31) // 32, dtype=BF, device="cuda"))
        out = dyn.moe_gated(x, Wn, off, pre=kept)
        assert not out[90:].any() and not kept.q[90:].any() and torch.isfinite(kept.scale[90:]).all()
        assert torch.isnan(out[5]).all() and torch.isfinite(out[:5]).all() and torch.isfinite(out[6:]).all() and torch.isnan(kept.scale[5]).all()
        W2 = dev(bf(g, E, K, n, std=0.1))
        pre = torch.randn(M, 2, n, device="cuda").to(BF)
        pre[90:] = float("nan")
        dpre, hidden = dyn.moe_gated_grad(dev(bf(g, M, K)), W2, off, pre)
        assert not dpre[90:].any() and not hidden[90:].any() and torch.isfinite(dpre).all()


def test_gradients_are_differences(dyn):
    """The backward pass against differences of the forward formula, in 64 bits: d/dg and d/du of sum dact f(g) u."""
    M, N, h = 40, 32, 24
    g = torch.Generator().manual_seed(9)
    dout, W, pre = bf(g, M, N), bf(g, 1, N, h, std=0.2), bf(g, M, 2, h)
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    dact = dout @ W[0]
    for gate in GATES:
        value = lambda p: dact * gate_of(gate, p[:, 0])[0] * p[:, 1]
        dpre, _ = dyn.moe_gated_grad(dev(dout), dev(W), off, dev(pre), gate=code(dyn, gate))
        for s in range(2):
            step = torch.zeros_like(pre)
            step[:, s] = 1e-6
            want = (value(pre + step) - value(pre - step)) / 2e-6
            within(dpre[:, s], want, stored(want, 1e-4 * (1 + dact.abs() * pre.abs().amax(1)), BF))


def test_no_rows(dyn):
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    W = torch.ones(2, 2, 8, 16, dtype=BF, device="cuda")
    pre = torch.empty(0, 2, 8, dtype=BF, device="cuda")
    assert dyn.moe_gated(torch.empty(0, 16, dtype=BF, device="cuda"), W, off, pre=pre).shape == (0, 8)
    assert dyn.moe_gated_grad(torch.empty(0, 16, dtype=BF, device="cuda"), torch.ones(2, 16, 8, dtype=BF, device="cuda"), off, pre)[0].shape == (0, 2, 8)


def plain_on_gpu(x, W1, off, perm, k, gate, dout=None, W2=None, restore=None):
    """The formulas in 64 bits on the GPU for sizes that the host takes long for; stands apart from the kernels' layouts."""
    M, h = len(perm), W1.shape[2]
    pre = torch.zeros(M, 2, h, dtype=F8, device="cuda")
    dact = torch.zeros(M, h, dtype=F8, device="cuda")
    for e in range(W1.shape[0]):
        a, b = int(off[e]), int(off[e + 1])
        if a == b:
            continue
        rows = x[(perm[a:b].long() // k)].double()
        pre[a:b, 0], pre[a:b, 1] = rows @ W1[e, 0].double().t(), rows @ W1[e, 1].double().t()
        if dout is not None:
            dact[a:b] = dout[a:b].double() @ W2[e].double()
    return pre, dact


@pytest.mark.parametrize("T,k,K,h,N,E,gate", [(8192, 2, 256, 512, 256, 8, "silu"), (16384, 1, 512, 1024, 512, 1, "gelu"), (4096, 4, 512, 1000, 264, 16, "silu"),
                                              (3000, 1, 1024, 2048, 512, 4, "gelu"), (20000, 2, 1024, 1024, 1024, 40, "silu")])
def test_large(dyn, T, k, K, h, N, E, gate):
    """Every kind of tile; errors relative to the tensor: 2^-8 for each rounding to bfloat16 (three tensors at most follow one another), scales' steps checked apart."""
    g = torch.Generator("cuda").manual_seed(T + E)
    M = T * k
    normal = lambda *shape, std=1.0: (torch.randn(*shape, generator=g, device="cuda") * std).to(BF)
    expert = (torch.rand(M, generator=g, device="cuda") ** 1.5 * E).long().clamp(max=E - 1)
    counts = torch.bincount(expert, minlength=E)
    off = torch.cat([torch.zeros(1, device="cuda", dtype=torch.long), counts.cumsum(0)]).int()
    perm = torch.argsort(expert, stable=True).int()
    x, W1, W2, dout = normal(T, K), normal(E, 2, h, K, std=K ** -0.5), normal(E, N, h, std=h ** -0.5), normal(M, N)
    pre, dact = plain_on_gpu(x, W1, off.cpu(), perm, k, gate, dout, W2)
    off_by = lambda a, b: float((a.double() - b).norm() / b.norm())
    f = gate_of(gate, pre[:, 0])[0]
    kept16 = torch.empty(M, 2, h, dtype=BF, device="cuda")
    kept8 = dyn.Rows8(torch.empty(M, 2, h, dtype=torch.int8, device="cuda"), torch.empty(M, 2, (h + 31) // 32, dtype=BF, device="cuda"))
    for keep in (None, kept16, kept8):
        out = dyn.moe_gated(x, W1, off, perm=perm, k=k, gate=code(dyn, gate), pre=keep)
        assert off_by(out, f * pre[:, 1]) < 2.0 ** -8
        assert float((out.double() - f * pre[:, 1]).abs().max()) <= float((f * pre[:, 1]).abs().max()) * 2.0 ** -8
    assert off_by(kept16, pre) < 2.0 ** -8
    stand = values(kept8.q, kept8.scale)
    half = kept8.scale.double().repeat_interleave(32, -1)[..., :h] / 2
    assert bool(((stand - pre).abs() <= half * (1 + 2.0 ** -15) + 1e-4).all())
    for keep, p in ((kept16, kept16.double()), (kept8, stand)):
        fp, slope = gate_of(gate, p[:, 0])[:2]
        dpre, hidden = dyn.moe_gated_grad(dout, W2, off, keep, gate=code(dyn, gate))
        assert off_by(dpre[:, 0], dact * p[:, 1] * slope) < 2.0 ** -8
        assert off_by(dpre[:, 1], dact * fp) < 2.0 ** -8
        assert off_by(hidden, fp * p[:, 1]) < 2.0 ** -8
        assert float((dpre[:, 1].double() - dact * fp).abs().max()) <= float((dact * fp).abs().max()) * 2.0 ** -8
