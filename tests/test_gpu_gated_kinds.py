"""The gated layer's larger tiles in both directions: 128 x 128 at sizes and addresses off their borders, 256 x 256 from and into 8 bits, with features and channels that end inside a
tile, groups without rows, and rows that no group has.  Every element against the formulas in 64 bits, with the bounds of tests/test_gpu_gated.py; the reference is computed on the GPU,
group by group."""
import pytest
import torch

from tests.operator_util import U32, stored
from tests.test_gpu_gated import BF, F8, code, dyn, gate_of  # noqa: F401
from tests.test_gpu_rows8 import blocks, values
from tests.tile_kinds import kind_of

pytestmark = pytest.mark.gpu


def inside(got, ref, bound, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    over = (got - ref).abs() - bound
    assert bool((over <= 0).all()), f"{what}: {int((over > 0).sum())} of {over.numel()} beyond their bound, worst by {float(over.max()):.3e}, first {torch.nonzero(over > 0)[0].tolist()}"


def groups(M, E, seed):
    """offsets: loads that differ, the second group empty, the last M // 50 rows nobody's"""
    g = torch.Generator().manual_seed(seed)
    share = torch.rand(E, generator=g) + 0.05
    if E > 1:
        share[1] = 0
    ends = (share.cumsum(0) / share.sum() * (M - M // 50)).long()
    return torch.cat([torch.zeros(1, dtype=torch.long), ends]).int()


def inputs(M, K, h, N, E, k=1, shift=0):
    """shift: elements that rows of activations begin behind a border of 16 bytes"""
    g = torch.Generator("cuda").manual_seed(M + K + h)

    def normal(*shape, std=1.0, shift=0):
        whole = torch.empty(shape[0], shape[-1] + shift, dtype=BF, device="cuda") if shift else torch.empty(shape, dtype=BF, device="cuda")
        whole.copy_(torch.randn(whole.shape, generator=g, device="cuda").mul_(std))
        return whole[:, shift:] if shift else whole
    perm = torch.randperm(M, generator=g, device="cuda").int() if k > 1 else None
    return normal((M + k - 1) // k, K, shift=shift), normal(E, 2, h, K, std=K ** -0.5), normal(M, N, shift=shift), normal(E, N, h, std=N ** -0.5), perm


def sums(rows_of, W, off):
    """rows W_e^T for W [E, n, K] and the bound of an fp32 sum's error, [M, n]"""
    M, n = int(off[-1]) if rows_of is None else len(rows_of), W.shape[1]
    y, err = torch.zeros(M, n, dtype=F8, device="cuda"), torch.zeros(M, n, dtype=F8, device="cuda")
    for e in range(W.shape[0]):
        a, b = int(off[e]), int(off[e + 1])
        if a < b:
            r, w = rows_of[a:b].double(), W[e].double().t().contiguous()
            y[a:b], err[a:b] = r @ w, (r.abs() @ w.abs()) * (W.shape[2] * 2 * U32)
    return y, err


def check_forward(dyn, M, K, h, N, E, k, gate, shift=0):  # noqa: F811
    x, W1, _, _, perm = inputs(M, K, h, N, E, k, shift)
    off = groups(M, E, M + h)
    rows = x if perm is None else x[perm.long() // k]
    pre, err = (t.view(M, 2, h) for t in sums(rows, W1.view(E, 2 * h, K), off))
    f, _, ef, _ = gate_of(gate, pre[:, 0])
    ref = f * pre[:, 1]
    bound = (1.13 * err[:, 0] + ef) * (pre[:, 1].abs() + err[:, 1]) + f.abs() * err[:, 1] + 2 * U32 * ref.abs()
    n, end = (h + 31) // 32, int(off[-1])
    kept16 = torch.full((M, 2, h), float("nan"), dtype=BF, device="cuda")
    kept8 = dyn.Rows8(torch.full((M, 2, h), 77, dtype=torch.int8, device="cuda"), torch.full((M, 2, n), 7.0, dtype=BF, device="cuda"))
    for what, keep in (("nothing", None), ("bf16", kept16), ("eight", kept8)):
        out = torch.full((M, h), float("nan"), dtype=BF, device="cuda")
        dyn.moe_gated(x, W1, off.cuda(), perm=perm, k=k, gate=code(dyn, gate), out=out, pre=keep)
        inside(out, ref, stored(ref, bound, BF), f"out, {what} kept")
        assert not out[end:].any(), what
        assert torch.equal(dyn.moe_gated(x, W1, off.cuda(), perm=perm, k=k, gate=code(dyn, gate), pre=keep), out)
    inside(kept16, pre, stored(pre, err, BF), "kept")
    assert not kept16[end:].any() and not kept8.q[end:].any() and torch.isfinite(kept8.scale).all()
    # the scale that the largest of a block may have, elements within half of it
    s = kept8.scale.double()
    up = lambda v: ((v.clamp(min=0).float() / 127).view(torch.int32) + 0xffff).bitwise_and(-0x10000).view(torch.float32).clamp(min=2.0 ** -126).double()
    largest, slack, room = blocks(pre.abs()).amax(-1), blocks(err).amax(-1), 1 + 4 * U32
    assert bool((s >= up((largest - slack) / room)).all()) and bool((s <= up((largest + slack) * room)).all())
    half = s.repeat_interleave(32, -1)[..., :h] / 2
    assert bool(((values(kept8.q, kept8.scale) - pre).abs() <= half * (1 + 2.0 ** -15) + err).all())


def check_grad(dyn, M, h, N, E, gate, eight, want_hidden=True, shift=0):  # noqa: F811
    _, _, dout, W2, _ = inputs(M, 8, h, N, E, 1, shift)
    off = groups(M, E, M + h)
    end = int(off[-1])
    pre = torch.randn(M, 2, h, generator=torch.Generator("cuda").manual_seed(h), device="cuda").mul_(2).to(BF)
    kept, stand = pre, pre.double()
    if eight:
        kept = dyn.Rows8(torch.empty(M, 2, h, dtype=torch.int8, device="cuda"), torch.empty(M, 2, (h + 31) // 32, dtype=BF, device="cuda"))
        for s in range(2):
            dyn.dynb_store8(pre[:, s], out=dyn.Rows8(kept.q[:, s], kept.scale[:, s]))
        stand = values(kept.q, kept.scale)
    dact, err = sums(dout, W2.transpose(1, 2).contiguous(), off)
    f, slope, ef, es = gate_of(gate, stand[:, 0])
    u = stand[:, 1]
    live = (torch.arange(M, device="cuda") < end)[:, None]
    dg, du, hid = dact * u * slope, dact * f, live * f * u
    bg = u.abs() * (err * (slope.abs() + es) + dact.abs() * es) + 4 * U32 * dg.abs()
    bu = err * (f.abs() + ef) + dact.abs() * ef + 4 * U32 * du.abs()
    dpre = torch.full((M, 2, h), float("nan"), dtype=BF, device="cuda")
    hidden = torch.full((M, h), float("nan"), dtype=BF, device="cuda") if want_hidden else None
    dyn.moe_gated_grad(dout, W2, off.cuda(), kept, gate=code(dyn, gate), dpre=dpre, hidden=hidden, want_hidden=want_hidden)
    inside(dpre[:, 0], dg, stored(dg, bg, BF), "gate")
    inside(dpre[:, 1], du, stored(du, bu, BF), "up")
    assert not dpre[end:].any()
    if want_hidden:
        inside(hidden, hid, stored(hid, live * (ef * u.abs() + 4 * U32 * hid.abs()), BF), "hidden")
        assert not hidden[end:].any()
    again = dyn.moe_gated_grad(dout, W2, off.cuda(), kept, gate=code(dyn, gate))
    assert torch.equal(again[0], dpre) and (hidden is None or torch.equal(again[1], hidden))


# 128 x 128 off the borders: nothing on them; the last chunk of 36 places; fewer than 8 features and places; an address alone; a place or a feature behind a tile
OFF = [(3001, 777, 1001, 777, 8, 0), (5000, 100, 1500, 100, 20, 0), (33000, 75, 7, 5, 8, 0), (3000, 512, 1024, 512, 4, 1), (2305, 65, 2049, 129, 3, 0), (40000, 193, 257, 1031, 16, 0)]


@pytest.mark.parametrize("M,K,h,N,E,shift", OFF)
@pytest.mark.parametrize("gate,k", [("silu", 1), ("gelu", 3)])
def test_128_off_borders_forward(dyn, M, K, h, N, E, shift, gate, k):  # noqa: F811
    assert kind_of(M, E, 2 * h, K) == "mid" and (K % 8 or h % 8 or shift)
    check_forward(dyn, M, K, h, N, E, k, gate, shift)


@pytest.mark.parametrize("M,K,h,N,E,shift", OFF)
@pytest.mark.parametrize("gate,eight,want_hidden", [("silu", False, True), ("gelu", True, True), ("silu", True, False)])
def test_128_off_borders_backward(dyn, M, K, h, N, E, shift, gate, eight, want_hidden):  # noqa: F811
    M = max(M, 16384 // ((h + 127) // 128) * 2 + 1)          # (half as many columns as forward)
    assert kind_of(M, E, h, N) == "mid" and (N % 8 or h % 8 or shift)
    check_grad(dyn, M, h, N, E, gate, eight, want_hidden, shift)


# 256 x 256: 8-bit rows on borders of 8 and of 16 bytes, 17 and 16 chunks, the last of 8, 40 and 64 places, two chunks, a tile of 8 features behind whole ones; one group
BIG = [(40000, 1032, 2056, 1032, 40, 1), (40000, 1000, 2064, 1064, 12, 2), (100000, 104, 4104, 104, 200, 1), (16384, 1024, 4096, 1024, 1, 1), (30001, 1088, 2312, 1096, 7, 4)]


@pytest.mark.parametrize("M,K,h,N,E,k", BIG)
@pytest.mark.parametrize("gate", ["silu", "gelu"])
def test_256_forward(dyn, M, K, h, N, E, k, gate):  # noqa: F811
    assert kind_of(M, E, 2 * h, K) == "big"
    check_forward(dyn, M, K, h, N, E, k, gate)


@pytest.mark.parametrize("M,K,h,N,E,k", BIG)
@pytest.mark.parametrize("gate,eight,want_hidden", [("silu", True, True), ("gelu", False, True), ("gelu", True, False)])
def test_256_backward(dyn, M, K, h, N, E, k, gate, eight, want_hidden):  # noqa: F811
    assert kind_of(M, E, h, N) == "big"
    check_grad(dyn, M, h, N, E, gate, eight, want_hidden)
