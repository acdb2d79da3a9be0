"""dynb_embed and dynb_embed_backward against plain sums in 64 bits.  Bounds: tests/operator_util.py; a row's gradient sums its tokens."""
import pytest
import torch

from tests.operator_util import gaps_untouched, stored, strided, within

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dyn():
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as d
    return d


def draw(T, V, kind, g):
    if kind == "same":                                   # one token over and over
        return torch.full((T,), V - 1, dtype=torch.int32)
    if kind == "zipf":
        p = torch.arange(1, V + 1, dtype=torch.float64) ** -1.1
        t = torch.randperm(V, generator=g)[torch.multinomial(p, T, replacement=True, generator=g)].int()
    else:
        t = torch.randint(V, (T,), generator=g).int()
    if kind == "padded" and T > 1:
        t[torch.rand(T, generator=g) < 0.3] = -1
        t[0], t[T - 1] = V, -2 ** 31                     # just outside, and far
    return t


SHAPES = [  # T, V, d, tokens
    (1, 1, 1, "same"), (1, 50000, 8, "any"), (3, 7, 5, "padded"), (37, 40, 64, "any"), (64, 512, 72, "padded"), (100, 5000, 257, "zipf"),
    (700, 33, 130, "same"), (1025, 2000, 512, "zipf"), (2049, 300, 96, "padded"), (4096, 70000, 32, "any"), (5000, 257, 1030, "zipf"),
    (9000, 511, 24, "same"), (20000, 1 << 16, 16, "zipf"), (20001, (1 << 18) + 1, 8, "padded"), (70000, 1000, 40, "zipf"),
]


@pytest.mark.parametrize("T,V,d,kind", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lookup(dyn, T, V, d, kind, dtype):
    g = torch.Generator().manual_seed(T + V)
    tokens = draw(T, V, kind, g)
    table = torch.randn(V, d, generator=g).to(DT[dtype])
    known = (tokens >= 0) & (tokens < V)
    ref = torch.where(known[:, None], table[torch.where(known, tokens, 0).long()].double() * 11.3137, 0.0)
    scale = torch.tensor(11.3137, dtype=torch.float32).double().item()
    ref = ref / 11.3137 * scale
    got = dyn.dynb_embed(tokens.cuda(), table.cuda(), scale=scale)
    within(got, ref, stored(ref, 2.0 ** -23 * ref.abs(), DT[dtype]))
    assert (got[~known.cuda()] == 0).all()


@pytest.mark.parametrize("T,V,d,kind", SHAPES)
@pytest.mark.parametrize("dtype,grad_dtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
def test_gradient(dyn, T, V, d, kind, dtype, grad_dtype):
    g = torch.Generator().manual_seed(T * 3 + V)
    tokens = draw(T, V, kind, g)
    dout = torch.randn(T, d, generator=g).to(DT[dtype])
    known = (tokens >= 0) & (tokens < V)
    at, rows = tokens[known].long(), dout[known].double()
    ref = torch.zeros(V, d, dtype=torch.float64).index_add_(0, at, rows) * 0.75
    mag = torch.zeros(V, d, dtype=torch.float64).index_add_(0, at, rows.abs()) * 0.75
    n = torch.bincount(at, minlength=V).double()[:, None]
    dtable = torch.full((V, d), float("nan"), dtype=DT[grad_dtype], device="cuda")
    args = (tokens.cuda(), dout.cuda(), V)
    got = dyn.dynb_embed_backward(*args, scale=0.75, dtable=dtable)
    within(got, ref, stored(ref, (n + 1) * 2.0 ** -23 * mag, DT[grad_dtype]))
    again = dyn.dynb_embed_backward(*args, scale=0.75, grad_dtype=dyn.DYNB_F32 if grad_dtype == "f32" else dyn.DYNB_BF16)
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,d", [(50, 30, 64), (50, 30, 61), (5000, 900, 128)])
@pytest.mark.parametrize("gap,offset", [(8, 0), (5, 0), (8, 1)])
def test_strides_and_addresses(dyn, dtype, T, V, d, gap, offset):
    g = torch.Generator().manual_seed(T)
    tokens, table, dout = draw(T, V, "padded", g).cuda(), torch.randn(V, d, generator=g).to(DT[dtype]).cuda(), torch.randn(T, d, generator=g)
    out, buf = strided(torch.zeros(T, d), gap, DT[dtype], offset)
    dyn.dynb_embed(tokens, table, scale=2.0, out=out)
    assert gaps_untouched(out, buf, offset) and torch.equal(out, dyn.dynb_embed(tokens, table, scale=2.0))
    dv, _ = strided(dout, gap, DT[dtype], offset)
    a, b = dyn.dynb_embed_backward(tokens, dv, V), dyn.dynb_embed_backward(tokens, dv.contiguous(), V)
    assert torch.allclose(a, b, rtol=1e-4, atol=1e-4)
    odd_table = torch.empty(V * d + 1, dtype=DT[dtype], device="cuda")[1:].view(V, d)
    odd_table.copy_(table)
    assert torch.equal(dyn.dynb_embed(tokens, odd_table, scale=2.0), dyn.dynb_embed(tokens, table, scale=2.0))
    odd_grad = torch.empty(V * d + 1, device="cuda")[1:].view(V, d)
    assert torch.allclose(dyn.dynb_embed_backward(tokens, dv, V, dtable=odd_grad), b, rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("T", [300, 9000])
@pytest.mark.parametrize("V,d", [(70001, 1024), (66003, 1029)])
def test_gradient_beyond_the_caches(dyn, T, V, d):
    """More than 256 MB of gradient: the rows without uses are stored another way."""
    g = torch.Generator().manual_seed(T + V)
    tokens = draw(T, V, "zipf", g).cuda()
    dout = torch.randn(T, d, generator=g).cuda()
    used, at = torch.unique(tokens, return_inverse=True)
    ref = torch.zeros(len(used), d, dtype=torch.float64).index_add_(0, at.cpu(), dout.double().cpu()) * 0.75
    mag = torch.zeros(len(used), d, dtype=torch.float64).index_add_(0, at.cpu(), dout.double().abs().cpu()) * 0.75
    n = torch.bincount(at.cpu()).double()[:, None]
    got = dyn.dynb_embed_backward(tokens, dout, V, scale=0.75, dtable=torch.full((V, d), float("nan"), device="cuda"))
    within(got[used.long()], ref, stored(ref, (n + 1) * 2.0 ** -23 * mag, torch.float32))
    unused = torch.ones(V, dtype=torch.bool, device="cuda")
    unused[used.long()] = False
    assert (got[unused] == 0).all()


@pytest.mark.parametrize("T", [300, 9000])
def test_gradient_of_the_most_rows(dyn, T):
    """2^27 rows, more than a workgroup for every eight of them has room in a launch."""
    V = 1 << 27
    g = torch.Generator().manual_seed(T)
    tokens = torch.randint(V, (T,), generator=g)
    tokens[:3] = torch.tensor([0, V - 1, V // 2 + 77])
    tokens[-100:] = tokens[5]
    dout = torch.randn(T, 1, generator=g)
    used, at = torch.unique(tokens, return_inverse=True)
    ref = torch.zeros(len(used), 1, dtype=torch.float64).index_add_(0, at, dout.double())
    mag = torch.zeros(len(used), 1, dtype=torch.float64).index_add_(0, at, dout.double().abs())
    n = torch.bincount(at).double()[:, None]
    got = dyn.dynb_embed_backward(tokens.int().cuda(), dout.cuda(), V, dtable=torch.full((V, 1), float("nan"), device="cuda"))
    within(got[used.cuda()], ref, stored(ref, (n + 1) * 2.0 ** -23 * mag, torch.float32))
    got[used.cuda()] = 0
    assert not got.any()


def test_what_is_not_finite_stays_in_its_row(dyn):
    tokens = torch.tensor([3, 1, 3, -1, 0, 9], dtype=torch.int32).cuda()
    dout = torch.ones(6, 64).cuda()
    dout[3], dout[5], dout[1] = float("nan"), float("inf"), float("nan")     # padding, out of range, token 1
    got = dyn.dynb_embed_backward(tokens, dout, 5)
    assert torch.isnan(got[1]).all() and (got[3] == 2).all() and (got[0] == 1).all() and (got[[2, 4]] == 0).all()


def test_no_tokens(dyn):
    tokens = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert dyn.dynb_embed(tokens, torch.ones(3, 8, device="cuda")).shape == (0, 8)
    grad = torch.full((3, 8), 5.0, device="cuda")
    assert (dyn.dynb_embed_backward(tokens, torch.ones(0, 8, device="cuda"), 3, dtable=grad) == 0).all()


def test_gradient_against_differences(dyn):
    g = torch.Generator().manual_seed(8)
    tokens, table, c = draw(200, 30, "padded", g), torch.randn(30, 16, generator=g), torch.randn(200, 16, generator=g)

    def f(tab):
        known = (tokens >= 0) & (tokens < 30)
        return float((c.double()[known] * tab[tokens[known].long()] * 1.5).sum())

    got = dyn.dynb_embed_backward(tokens.cuda(), c.cuda(), 30, scale=1.5).double().cpu()
    for _ in range(4):
        p = torch.randn(30, 16, generator=g, dtype=torch.float64)
        assert abs((f(table + 1e-3 * p) - f(table - 1e-3 * p)) / 2e-3 - float((got * p).sum())) <= 1e-5 * float((got * p).abs().sum())


def test_other_streams_and_graphs(dyn):
    g = torch.Generator().manual_seed(5)
    for T, V in ((900, 700), (6000, 3000)):
        tokens, table, dout = draw(T, V, "zipf", g).cuda(), torch.randn(V, 128, generator=g).cuda(), torch.randn(T, 128, generator=g).cuda()
        out, grad = torch.empty(T, 128, device="cuda"), torch.empty(V, 128, device="cuda")
        ws = torch.empty(dyn.dynb_embed_backward_workspace_bytes(T, V, 128, dyn.DYNB_F32), dtype=torch.uint8, device="cuda")

        def step(stream=None):
            dyn.dynb_embed(tokens, table, scale=3.0, out=out, stream=stream)
            dyn.dynb_embed_backward(tokens, dout, V, scale=3.0, dtable=grad, workspace=ws, stream=stream)

        step()
        torch.cuda.synchronize()
        ref = [out.clone(), grad.clone()]
        side = torch.cuda.Stream()
        out.fill_(1), grad.fill_(1)
        torch.cuda.synchronize()
        step(side)
        side.synchronize()
        assert torch.equal(out, ref[0]) and torch.equal(grad, ref[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(3):
            out.fill_(1), grad.fill_(1), ws.fill_(255)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref[0]) and torch.equal(grad, ref[1])
