"""dynb_layer_norm and dynb_layer_norm_backward against plain forms in 64 bits.

Bounds, u = 2^-24, sums of n numbers in fp32 off by n u times the sum of their magnitudes: the mean by (d + 1) u mean|x| =: e; the variance,
a sum of squares of differences from that mean, by a factor 1 +- (d + 6) u and by e^2; r by half of that, relative.  So y is off by
|gamma| (r e + |h| ((d + 16) u + (r e)^2)) + 4 u (|h gamma| + |beta|), and half a unit of what it is stored in.  The backward pass takes
mean and rstd as they are: every term of dx by (d + 16) u of its magnitude, the sums over the rows by (T + 16) u."""
import pytest
import torch

from tests.operator_util import gaps_untouched, stored, strided, within

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dyn():
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as d
    return d


def forward(x, gamma, beta, eps):
    d = x.shape[1]
    m = x.mean(1, keepdim=True)
    r = ((x - m).square().mean(1, keepdim=True) + eps).rsqrt()
    h = (x - m) * r
    e = (d + 1) * U * x.abs().mean(1, keepdim=True)
    bound = gamma.abs() * (r * e + h.abs() * ((d + 16) * U + (r * e) ** 2)) + 4 * U * ((h * gamma).abs() + beta.abs())
    return h * gamma + beta, bound, m[:, 0], e[:, 0], r[:, 0], ((d + 16) * U + (r * e) ** 2)[:, 0] * r[:, 0]


SHAPES = [(1, 1), (3, 2), (5, 7), (1, 64), (37, 512), (9, 513), (64, 777), (130, 1024), (33, 1032), (20, 2048), (7, 2050), (65, 4096), (5, 8192),
          (4, 8200), (3, 16384), (2, 20001), (3000, 64), (5001, 96), (2048, 256)]


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("params", [True, False])
def test_forward(dyn, T, d, dtype, params):
    g = torch.Generator().manual_seed(T * 5 + d)
    x = (torch.randn(T, d, generator=g) * (0.1 + 3 * torch.rand(T, 1, generator=g)) + 2 * torch.randn(T, 1, generator=g)).to(DT[dtype])
    gamma = torch.randn(d, generator=g) if params else None
    beta = torch.randn(d, generator=g) if params else None
    eps = torch.tensor(1e-5, dtype=torch.float32).double().item()
    one, zero = torch.ones(d, dtype=torch.float64), torch.zeros(d, dtype=torch.float64)
    y, bound, m, em, r, er = forward(x.double(), gamma.double() if params else one, beta.double() if params else zero, eps)
    dev = lambda t: None if t is None else t.cuda()
    got, mean, rstd = dyn.dynb_layer_norm(x.cuda(), dev(gamma), dev(beta), eps=1e-5, want_stats=True)
    within(mean, m, em + U * m.abs(), "mean")
    within(rstd, r, er + 4 * U * r, "rstd")
    within(got, y, stored(y, bound, DT[dtype]), "y")
    assert torch.equal(got, dyn.dynb_layer_norm(x.cuda(), dev(gamma), dev(beta), eps=1e-5))


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("params", [True, False])
def test_backward(dyn, T, d, dtype, params):
    g = torch.Generator().manual_seed(T * 7 + d)
    x = (torch.randn(T, d, generator=g) * (0.5 + torch.rand(T, 1, generator=g)) + torch.randn(T, 1, generator=g)).to(DT[dtype])
    dy = (torch.randn(T, d, generator=g) * 0.1).to(DT[dtype])
    gamma = torch.randn(d, generator=g) if params else None
    xd, dyd = x.double(), dy.double()
    mean = xd.mean(1).float()
    rstd = ((xd - xd.mean(1, keepdim=True)).square().mean(1) + 1e-5).rsqrt().float()
    h = (xd - mean.double()[:, None]) * rstd.double()[:, None]
    gr = dyd * (gamma.double() if params else 1.0)
    r, gh = rstd.double()[:, None], gr * h
    dx = r * (gr - gr.mean(1, keepdim=True) - h * gh.mean(1, keepdim=True))
    bx = r * (gr.abs() + gr.abs().mean(1, keepdim=True) + h.abs() * gh.abs().mean(1, keepdim=True)) * (d + 16) * U
    got, dgamma, dbeta = dyn.dynb_layer_norm_backward(dy.cuda(), x.cuda(), gamma.cuda() if params else None, mean.cuda(), rstd.cuda())
    within(got, dx, stored(dx, bx, DT[dtype]), "dx")
    within(dgamma, (dyd * h).sum(0), (T + 16) * U * (dyd * h).abs().sum(0) + 1e-38, "dgamma")
    within(dbeta, dyd.sum(0), (T + 16) * U * dyd.abs().sum(0) + 1e-38, "dbeta")
    again = dyn.dynb_layer_norm_backward(dy.cuda(), x.cuda(), gamma.cuda() if params else None, mean.cuda(), rstd.cuda())
    assert torch.equal(got, again[0]) and torch.equal(dgamma, again[1]) and torch.equal(dbeta, again[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d", [(40, 128), (40, 127), (9, 2048), (3, 9000)])
@pytest.mark.parametrize("gap,offset", [(8, 0), (3, 0), (8, 1)])
def test_strides_addresses_and_in_place(dyn, dtype, T, d, gap, offset):
    g = torch.Generator().manual_seed(T)
    x, dy, gamma = torch.randn(T, d, generator=g).to(DT[dtype]).cuda(), torch.randn(T, d, generator=g).to(DT[dtype]).cuda(), torch.randn(d, generator=g).cuda()
    ref, mean, rstd = dyn.dynb_layer_norm(x, gamma, None, want_stats=True)
    ref_b = dyn.dynb_layer_norm_backward(dy, x, gamma, mean, rstd)
    xv, xbuf = strided(x, gap, DT[dtype], offset)
    dv, dbuf = strided(dy, gap, DT[dtype], offset)
    out, buf = strided(torch.zeros(T, d), gap, DT[dtype], offset)
    close = lambda a, b: torch.allclose(a.float(), b.float(), rtol=2.0 ** -7, atol=1e-4)     # (another kernel's order of summation)
    assert close(dyn.dynb_layer_norm(xv, gamma, None, out=out), ref) and gaps_untouched(out, buf, offset)
    got = dyn.dynb_layer_norm_backward(dv, xv, gamma, mean, rstd, dx=out)
    assert all(close(a, b) for a, b in zip(got, ref_b)) and gaps_untouched(out, buf, offset)
    got = dyn.dynb_layer_norm_backward(dv, xv, gamma, mean, rstd, dx=dv)                     # into dy
    assert close(got[0], ref_b[0]) and gaps_untouched(dv, dbuf, offset)
    assert close(dyn.dynb_layer_norm(xv, gamma, None, out=xv), ref) and gaps_untouched(xv, xbuf, offset)


def test_constant_rows_large_means_and_what_is_not_finite(dyn):
    x = torch.zeros(6, 256)
    x[0] = 5.0                                           # no variance: eps decides
    x[1] = torch.randn(256, generator=torch.Generator().manual_seed(1)) + 3e4     # a mean that would drown the variance of E[x^2] - m^2
    x[2] = 1e19                                          # squares of x, though not of x - m, leave fp32
    x[3, 7] = float("nan")
    x[4, 9] = float("inf")
    y, mean, rstd = dyn.dynb_layer_norm(x.cuda(), want_stats=True)
    eps = torch.tensor(1e-5).double().item()
    ref, bound, m, em, r, er = forward(x[:2].double(), torch.ones(256, dtype=torch.float64), torch.zeros(256, dtype=torch.float64), eps)
    within(y[:2], ref, stored(ref, bound, torch.float32))
    within(rstd[:2], r, er + 4 * U * r)
    assert torch.isfinite(y[2]).all() and torch.isnan(y[3]).all() and not torch.isfinite(y[4]).any()
    assert (y[5] == 0).all() and torch.isfinite(rstd[5])


def test_no_rows(dyn):
    e = torch.empty(0, device="cuda")
    x = torch.ones(0, 8, device="cuda")
    assert dyn.dynb_layer_norm(x).shape == (0, 8)
    dx, dgamma, dbeta = dyn.dynb_layer_norm_backward(x, x, None, e, e)
    assert dx.shape == (0, 8) and (dgamma == 0).all() and (dbeta == 0).all()


def test_gradient_against_differences(dyn):
    g = torch.Generator().manual_seed(8)
    x, c, gamma, beta = (torch.randn(*s, generator=g, dtype=torch.float64).float() for s in ((30, 48), (30, 48), (48,), (48,)))
    eps = 1e-5

    def f(x, gamma, beta):
        m = x.mean(1, keepdim=True)
        return float((c.double() * ((x - m) * ((x - m).square().mean(1, keepdim=True) + eps).rsqrt() * gamma + beta)).sum())

    _, mean, rstd = dyn.dynb_layer_norm(x.cuda(), gamma.cuda(), beta.cuda(), eps=eps, want_stats=True)
    grads = [t.double().cpu() for t in dyn.dynb_layer_norm_backward(c.cuda(), x.cuda(), gamma.cuda(), mean.cuda(), rstd.cuda())]
    at = [x.double(), gamma.double(), beta.double()]
    for i in range(3):
        for _ in range(3):
            p, h = torch.randn(at[i].shape, generator=g, dtype=torch.float64), 1e-5
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * p, at[i] - h * p
            assert abs((f(*up) - f(*down)) / (2 * h) - float((grads[i] * p).sum())) <= 1e-5 * float((grads[i] * p).abs().sum()) + 1e-6


def test_other_streams_and_graphs(dyn):
    g = torch.Generator().manual_seed(5)
    T, d = 3000, 512
    x, dy, gamma = torch.randn(T, d, generator=g).cuda(), torch.randn(T, d, generator=g).cuda(), torch.randn(d, generator=g).cuda()
    ws = torch.empty(dyn.dynb_layer_norm_backward_workspace_bytes(T, d, dyn.DYNB_F32), dtype=torch.uint8, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)

    def step(stream=None):
        _, mean, rstd = dyn.dynb_layer_norm(x, gamma, out=y, want_stats=True, stream=stream)
        return (y,) + dyn.dynb_layer_norm_backward(dy, x, gamma, mean, rstd, dx=dx, workspace=ws, stream=stream)

    ref = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y.fill_(1), dx.fill_(1)
    torch.cuda.synchronize()
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for t in got:
            t.fill_(1)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
