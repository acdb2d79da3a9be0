"""moe_product, moe_product_grad_input and moe_product_grad_weight against plain products in 64 bits, expert by expert.

Bounds: tests/operator_util.py; a product sums K, N or the group's rows."""
import numpy as np
import pytest
import torch

from tests.operator_util import gaps_untouched, stored, strided, within

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def dyn():
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as d
    return d


def bf(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * std).to(BF).double()


def dev(t, dtype=BF):
    return t.to(dtype).cuda()


def counts_of(kind, M, E, g):
    """Rows of every expert: the shapes that loads take."""
    c = [0] * E
    if kind == "last":                                   # all in the last one
        c[E - 1] = M
    elif kind == "first":
        c[0] = M
    elif kind == "ones":                                 # one row each, as far as they go
        for r in range(M):
            c[r % E] += 1
    elif kind == "tail":                                 # a third of the rows are nobody's
        for r in range(M - M // 3):
            c[int(torch.randint(E, (1,), generator=g))] += 1
    else:                                                # skewed, some empty
        for r in range(M):
            c[min(E - 1, int(E * torch.rand((1,), generator=g).item() ** 3))] += 1
        if E > 2 and kind == "holes":
            c[E // 2] += c[0]
            c[0] = 0
    return c


SHAPES = [  # M, K, N, E, loads
    (1, 1, 1, 1, "first"),
    (5, 3, 2, 4, "skew"),
    (70, 40, 24, 3, "holes"),
    (65, 64, 64, 1, "first"),
    (64, 72, 136, 5, "tail"),
    (130, 64, 128, 9, "last"),
    (257, 129, 131, 7, "skew"),          # odd: no fast kernel
    (300, 128, 192, 300, "ones"),
    (74, 512, 256, 64, "skew"),          # a few tokens
    (513, 256, 320, 6, "holes"),
    (1000, 192, 520, 11, "skew"),
    (1300, 320, 264, 3, "tail"),
    (700, 8, 16, 2, "skew"),
    (2100, 576, 640, 2, "skew"),
    (4500, 256, 256, 1, "first"),        # one crowded expert: its gradient's sum is long
    (5000, 320, 192, 130, "skew"),
]


@pytest.mark.parametrize("M,K,N,E,loads", SHAPES)
@pytest.mark.parametrize("gathered", [False, True])
def test_forward(dyn, M, K, N, E, loads, gathered):
    g = torch.Generator().manual_seed(M * 7 + K)
    counts = counts_of(loads, M, E, g)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    k = 3 if gathered else 1
    n_rows = (M + k - 1) // k if gathered else M
    x, W = bf(g, n_rows, K), bf(g, E, N, K, std=K ** -0.5)
    perm = torch.randperm(M, generator=g).int() if gathered else None
    rows = x[perm.long() // k] if gathered else x
    ref, mag = torch.zeros(M, N, dtype=torch.float64), torch.zeros(M, N, dtype=torch.float64)
    for e in range(E):
        a, b = off[e], off[e + 1]
        ref[a:b], mag[a:b] = rows[a:b] @ W[e].t(), rows[a:b].abs() @ W[e].abs().t()
    for relu in (False, True):
        want = ref.clamp(min=0) if relu else ref
        out = torch.full((M, N), float("nan"), dtype=BF, device="cuda")
        got = dyn.moe_product(dev(x), dev(W), torch.from_numpy(off).cuda(), perm=perm.cuda() if gathered else None, k=k, relu=relu, out=out)
        assert got is out
        within(got, want, stored(want, K * 2.0 ** -23 * mag, BF), f"relu {relu}")


@pytest.mark.parametrize("M,K,N,E,loads", SHAPES)
@pytest.mark.parametrize("masked", [False, True])
def test_grad_input(dyn, M, K, N, E, loads, masked):
    g = torch.Generator().manual_seed(M * 11 + K)
    counts = counts_of(loads, M, E, g)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    dout, W = bf(g, M, N), bf(g, E, N, K, std=N ** -0.5)
    act = bf(g, M, K)
    act[torch.rand(M, K, generator=g) < 0.3] = 0.0
    act[0, 0] = -0.0
    ref, mag = torch.zeros(M, K, dtype=torch.float64), torch.zeros(M, K, dtype=torch.float64)
    for e in range(E):
        a, b = off[e], off[e + 1]
        ref[a:b], mag[a:b] = dout[a:b] @ W[e], dout[a:b].abs() @ W[e].abs()
    if masked:
        ref = torch.where(act > 0, ref, 0.0)
        act[-1, -1] = float("nan")                       # not above 0
        ref[-1, -1] = 0.0
    out = torch.full((M, K), float("nan"), dtype=BF, device="cuda")
    got = dyn.moe_product_grad_input(dev(dout), dev(W), torch.from_numpy(off).cuda(), act=dev(act) if masked else None, out=out)
    within(got, ref, stored(ref, N * 2.0 ** -23 * mag, BF) * (ref != 0) if masked else stored(ref, N * 2.0 ** -23 * mag, BF))


@pytest.mark.parametrize("M,K,N,E,loads", SHAPES)
@pytest.mark.parametrize("gathered", [False, True])
@pytest.mark.parametrize("grad_dtype", ["f32", "bf16"])
def test_grad_weight(dyn, M, K, N, E, loads, gathered, grad_dtype):
    g = torch.Generator().manual_seed(M * 13 + K)
    counts = counts_of(loads, M, E, g)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    k = 2 if gathered else 1
    n_rows = (M + k - 1) // k if gathered else M
    dout, x = bf(g, M, N), bf(g, n_rows, K)
    perm = torch.randperm(M, generator=g).int() if gathered else None
    rows = x[perm.long() // k] if gathered else x
    ref, bound = torch.zeros(E, N, K, dtype=torch.float64), torch.zeros(E, N, K, dtype=torch.float64)
    dt = torch.float32 if grad_dtype == "f32" else BF
    for e in range(E):
        a, b = off[e], off[e + 1]
        ref[e] = dout[a:b].t() @ rows[a:b]
        bound[e] = stored(ref[e], (b - a) * 2.0 ** -23 * (dout[a:b].abs().t() @ rows[a:b].abs()), dt)
    dW = torch.full((E, N, K), float("nan"), dtype=dt, device="cuda")
    args = (dev(dout), dev(x), torch.from_numpy(off).cuda())
    got = dyn.moe_product_grad_weight(*args, perm=perm.cuda() if gathered else None, k=k, dW=dW)
    within(got, ref, bound)
    again = dyn.moe_product_grad_weight(*args, perm=perm.cuda() if gathered else None, k=k, grad_dtype=dyn.DYNB_F32 if grad_dtype == "f32" else dyn.DYNB_BF16)
    assert torch.equal(got, again)


@pytest.mark.parametrize("M,K,N,E", [(150, 64, 128, 4), (150, 62, 130, 4), (600, 128, 256, 2)])
@pytest.mark.parametrize("gap,offset", [(8, 0), (64, 8), (3, 0), (8, 1)])
def test_strides_and_addresses(dyn, M, K, N, E, gap, offset):
    """Rows apart, rows off the 16-byte borders: nothing between them is read or written."""
    g = torch.Generator().manual_seed(M + gap)
    off = np.concatenate([[0], np.cumsum(counts_of("skew", M, E, g))]).astype(np.int32)
    o = torch.from_numpy(off).cuda()
    x, W, dout = bf(g, M, K), bf(g, E, N, K), bf(g, M, N)
    xv, _ = strided(x, gap, BF, offset)
    dv, _ = strided(dout, gap, BF, offset)
    av, _ = strided(x, gap, BF, offset)
    for name, got, plain, shape in [
            ("product", lambda out: dyn.moe_product(xv, dev(W), o, out=out), lambda: dyn.moe_product(dev(x), dev(W), o), (M, N)),
            ("grad_input", lambda out: dyn.moe_product_grad_input(dv, dev(W), o, act=av, out=out),
             lambda: dyn.moe_product_grad_input(dev(dout), dev(W), o, act=dev(x)), (M, K))]:
        out, buf = strided(torch.zeros(shape), gap, BF, offset)
        got(out)
        ref = plain().double()
        assert gaps_untouched(out, buf, offset), name
        # both are within half a unit of the same sum, whatever kernels they ran on
        assert ((out.double() - ref).abs() <= 2.0 ** -7 * ref.abs() + 1e-3).all(), name
    a, b = dyn.moe_product_grad_weight(dv, xv, o), dyn.moe_product_grad_weight(dev(dout), dev(x), o)
    assert torch.allclose(a, b, rtol=1e-4, atol=1e-2)


def test_rows_of_infinities_stay_with_their_rows(dyn):
    """What is not finite in one row, or in one expert's matrix, shows nowhere else: ragged tiles read past no border."""
    g = torch.Generator().manual_seed(3)
    M, K, N, E = 200, 64, 128, 4
    off = torch.tensor([0, 50, 50, 131, 200], dtype=torch.int32)
    x, W, dout = bf(g, M, K), bf(g, E, N, K), bf(g, M, N)
    clean = dyn.moe_product(dev(x), dev(W), off.cuda())
    clean_in = dyn.moe_product_grad_input(dev(dout), dev(W), off.cuda())
    clean_w = dyn.moe_product_grad_weight(dev(dout), dev(x), off.cuda())
    for bad in (float("inf"), float("nan")):
        xb, db, Wb = x.clone(), dout.clone(), W.clone()
        xb[60], db[60] = bad, bad                        # of expert 2
        Wb[1] = bad                                      # an empty expert
        got = dyn.moe_product(dev(xb), dev(Wb), off.cuda())
        keep = torch.arange(M) != 60
        assert torch.equal(got[keep.cuda()], clean[keep.cuda()]) and not torch.isfinite(got[60]).any()
        got = dyn.moe_product_grad_input(dev(db), dev(Wb), off.cuda())
        assert torch.equal(got[keep.cuda()], clean_in[keep.cuda()]) and not torch.isfinite(got[60]).any()
        got = dyn.moe_product_grad_weight(dev(db), dev(x), off.cuda())
        assert torch.equal(got[[0, 1, 3]], clean_w[[0, 1, 3]]) and not torch.isfinite(got[2]).any()
    got = dyn.moe_product(dev(torch.full((M, K), float("nan"))), dev(W), off.cuda(), relu=True)
    assert torch.isnan(got).all()                        # ReLU keeps a NaN


def test_no_rows(dyn):
    o = torch.zeros(4, dtype=torch.int32, device="cuda")
    W = torch.ones((3, 16, 8), dtype=BF, device="cuda")
    x = torch.ones((0, 8), dtype=BF, device="cuda")
    d = torch.ones((0, 16), dtype=BF, device="cuda")
    assert dyn.moe_product(x, W, o).shape == (0, 16) and dyn.moe_product_grad_input(d, W, o).shape == (0, 8)
    dW = torch.full((3, 16, 8), 5.0, device="cuda")
    assert (dyn.moe_product_grad_weight(d, x, o, dW=dW) == 0).all()


def test_gradients_against_differences(dyn):
    """sum(c * ReLU-layer(x)) moved along random directions, in differences of the 64-bit forward pass, against the gradients' products."""
    g = torch.Generator().manual_seed(9)
    M, K, N, E = 120, 64, 96, 5
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(counts_of("skew", M, E, g))]).astype(np.int32))
    x, W, c = bf(g, M, K).clamp(min=0), bf(g, E, N, K), bf(g, M, N)

    def f(x, W):
        return sum(float((c[a:b] * (x[a:b] @ W[e].t())).sum()) for e, (a, b) in enumerate(zip(off[:-1].tolist(), off[1:].tolist())))

    dx = dyn.moe_product_grad_input(dev(c), dev(W), off.cuda(), act=dev(x)).double().cpu()
    dW = dyn.moe_product_grad_weight(dev(c), dev(x), off.cuda()).double().cpu()
    for _ in range(4):
        px, pW, h = torch.randn(M, K, generator=g, dtype=torch.float64) * (x > 0), torch.randn(E, N, K, generator=g, dtype=torch.float64), 1e-4
        num_x, num_w = (f(x + h * px, W) - f(x - h * px, W)) / (2 * h), (f(x, W + h * pW) - f(x, W - h * pW)) / (2 * h)
        # dx is stored in bfloat16: every element off by 2^-8 of itself at most
        assert abs(num_x - float((dx * px).sum())) <= 2.0 ** -8 * float((dx * px).abs().sum()) + 1e-6 * abs(num_x) + 1e-6
        assert abs(num_w - float((dW * pW).sum())) <= 1e-5 * float((dW * pW).abs().sum())


def test_other_streams_and_graphs(dyn):
    g = torch.Generator().manual_seed(4)
    M, K, N, E = 900, 128, 192, 5
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(counts_of("skew", M, E, g))]).astype(np.int32)).cuda()
    x, W, dout = dev(bf(g, M, K)), dev(bf(g, E, N, K)), dev(bf(g, M, N))
    out, din, dW = torch.empty_like(dout), torch.empty_like(x), torch.empty((E, N, K), device="cuda")
    ws = torch.empty(dyn.moe_product_grad_weight_workspace_bytes(M, K, N, E), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        dyn.moe_product(x, W, off, relu=True, out=out, stream=stream)
        dyn.moe_product_grad_input(dout, W, off, act=x, out=din, stream=stream)
        dyn.moe_product_grad_weight(dout, x, off, dW=dW, workspace=ws, stream=stream)

    step()
    torch.cuda.synchronize()
    ref = [t.clone() for t in (out, din, dW)]
    side = torch.cuda.Stream()
    for t in (out, din, dW):
        t.fill_(3)
    torch.cuda.synchronize()
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, (out, din, dW)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (out, din, dW):
            t.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, (out, din, dW)))


def test_rows_beyond_four_gigabytes(dyn):
    """Rows a megaelement apart: offsets into x, dout and the results pass 32 bits, whether rows are gathered or not."""
    g = torch.Generator().manual_seed(12)
    M, K, N, E, pitch = 2100, 64, 72, 3, 1 << 20
    off = torch.tensor([0, 700, 701, M], dtype=torch.int32).cuda()
    buf = torch.empty(M * pitch, dtype=BF, device="cuda")
    wide = buf.view(M, pitch)
    x, dout, W = dev(bf(g, M, K)), dev(bf(g, M, N)), dev(bf(g, E, N, K))
    perm = torch.randperm(2 * M, generator=g).int().cuda()
    off2 = (off * 2).contiguous()
    wide[:, 128:128 + K], wide[:, 256:256 + N] = x, dout
    xv, dv = wide[:, 128:128 + K], wide[:, 256:256 + N]
    # (the dense tensors run another kernel where the offsets decide; products of the same numbers, rounded once each)
    close = lambda a, b: torch.allclose(a.float(), b.float(), rtol=2.0 ** -7, atol=1e-3)
    assert close(dyn.moe_product(xv, W, off), dyn.moe_product(x, W, off))
    assert close(dyn.moe_product(xv, W, off2, perm=perm, k=2), dyn.moe_product(x, W, off2, perm=perm, k=2))
    assert close(dyn.moe_product_grad_input(dv, W, off, act=xv), dyn.moe_product_grad_input(dout, W, off, act=x))
    assert torch.allclose(dyn.moe_product_grad_weight(dv, xv, off), dyn.moe_product_grad_weight(dout, x, off), rtol=1e-4, atol=1e-2)
    d2 = dev(bf(g, 2 * M, N))
    assert torch.allclose(dyn.moe_product_grad_weight(d2, xv, off2, perm=perm, k=2), dyn.moe_product_grad_weight(d2, x, off2, perm=perm, k=2), rtol=1e-4, atol=1e-2)
    out = wide[:, 512:512 + N]
    dyn.moe_product(x, W, off, out=out)
    assert close(out, dyn.moe_product(x, W, off))


@pytest.mark.parametrize("M,K,N,E,loads", [(16384, 2048, 1928, 20, "skew"), (20001, 2056, 2048, 30, "holes"), (16384, 1024, 1024, 20, "skew"), (13000, 2048, 1032, 30, "holes"), (9000, 136, 200, 400, "skew"), (30000, 264, 72, 2, "tail")])
def test_many_rows_of_every_kind_of_tile(dyn, M, K, N, E, loads):
    """Sizes at which every kind of tile runs (crowded experts on the largest), against products in 64 bits on the GPU."""
    g = torch.Generator().manual_seed(M)
    r = np.random.Generator(np.random.Philox(key=[M, K]))
    share = r.random(E) ** 3
    if loads == "holes":
        share[::3] = 0
    counts = np.bincount(r.choice(E, M - M // 3 if loads == "tail" else M, p=share / share.sum()), minlength=E)
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    at = off.tolist()
    x, W, dout = dev(bf(g, (M + 1) // 2, K)), dev(bf(g, E, N, K, std=K ** -0.5)), dev(bf(g, M, N, std=N ** -0.5))
    perm, act = torch.randperm(M, generator=g).int().cuda(), dev(bf(g, M, K))
    rows = x.double()[perm.long() // 2]
    fwd, gin = torch.zeros(M, N, dtype=torch.float64, device="cuda"), torch.zeros(M, K, dtype=torch.float64, device="cuda")
    bf_, bi = torch.zeros_like(fwd), torch.zeros_like(gin)
    gw, bw = torch.zeros(E, N, K, dtype=torch.float64, device="cuda"), torch.zeros(E, N, K, dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b, w, d = at[e], at[e + 1], W[e].double(), dout[at[e]:at[e + 1]].double()
        fwd[a:b], bf_[a:b] = rows[a:b] @ w.t(), K * 2.0 ** -23 * (rows[a:b].abs() @ w.abs().t())
        gin[a:b], bi[a:b] = (d @ w) * (act[a:b] > 0), N * 2.0 ** -23 * (d.abs() @ w.abs())
        gw[e], bw[e] = d.t() @ rows[a:b], (b - a) * 2.0 ** -23 * (d.abs().t() @ rows[a:b].abs())
    cpu = lambda t: t.cpu()
    got = dyn.moe_product(x, W, off, perm=perm, k=2, relu=True, out=torch.full((M, N), float("nan"), dtype=BF, device="cuda"))
    within(got, cpu(fwd.clamp(min=0)), cpu(stored(fwd.clamp(min=0), bf_, BF)), "forward")
    got = dyn.moe_product_grad_input(dout, W, off, act=act, out=torch.full((M, K), float("nan"), dtype=BF, device="cuda"))
    within(got, cpu(gin), cpu(stored(gin, bi, BF)), "input's gradient")
    for dt in (torch.float32, BF):
        got = dyn.moe_product_grad_weight(dout, x, off, perm=perm, k=2, dW=torch.full((E, N, K), float("nan"), dtype=dt, device="cuda"))
        within(got, cpu(gw), cpu(stored(gw, bw, dt)), "weights' gradient")
        assert torch.equal(got, dyn.moe_product_grad_weight(dout, x, off, perm=perm, k=2, dW=torch.empty_like(got)))
