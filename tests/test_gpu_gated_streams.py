"""The gated layer and the rows in 8 bits on other streams, in graphs, on memory that earlier work still writes, and two calls at once."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def dyn():
    assert torch.cuda.is_available()
    import paper_1707_02402_amd as d
    return d


def room8(dyn, *shape):
    return dyn.Rows8(torch.zeros(shape, dtype=torch.int8, device="cuda"), torch.zeros((*shape[:-1], (shape[-1] + 31) // 32), dtype=BF, device="cuda"))


def calls(dyn, K=96, h=160, M=1500, E=7, seed=1):
    """name -> f(stream) -> tensors; everything that is written is the call's own"""
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(BF)
    x, W1, W2, dout = normal(M, K), normal(E, 2, h, K) * K ** -0.5, normal(E, K, h) * K ** -0.5, normal(M, K)
    off = torch.tensor([0, 0, 130, 700, 701, 1100, 1300, M - 20], dtype=torch.int32, device="cuda")
    kept16, gamma = normal(M, 2, h), torch.ones(K, device="cuda")
    kept8 = room8(dyn, M, 2, h)
    dyn.moe_gated(x, W1, off, pre=kept8)
    xs = dyn.dynb_store8(x)
    _, mean, rstd = dyn.dynb_layer_norm(x, gamma, want_stats=True)

    def with_pre(stream):
        own = room8(dyn, M, 2, h) if stream is None else with_pre.own
        return [dyn.moe_gated(x, W1, off, gate=dyn.MOE_GATE_GELU, pre=own, stream=stream), own.q, own.scale]
    with_pre.own = room8(dyn, M, 2, h)
    return dict(gated=lambda s: [dyn.moe_gated(x, W1, off, stream=s)], gated_pre8=with_pre, grad16=lambda s: list(dyn.moe_gated_grad(dout, W2, off, kept16, stream=s)),
                grad8=lambda s: list(dyn.moe_gated_grad(dout, W2, off, kept8, stream=s)), store8=lambda s: list(dyn.dynb_store8(x, stream=s)), load8=lambda s: [dyn.dynb_load8(xs, stream=s)],
                norm8=lambda s: list(dyn.dynb_layer_norm_backward(dout, xs, gamma, mean, rstd, stream=s)))


NAMES = ["gated", "gated_pre8", "grad16", "grad8", "store8", "load8", "norm8"]


@pytest.mark.parametrize("name", NAMES)
def test_other_streams_and_memory_in_use(dyn, name):
    call = calls(dyn)[name]
    want = [t.clone() for t in call(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (512, 512, 4096, 16384, 65536, 1 << 18, 1 << 19, 1 << 19, 1 << 20, 1 << 20, 1 << 21)]
    for _ in range(40):
        for t in busy:
            t.fill_(0x55)
    del busy, t
    got = call(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    with torch.cuda.stream(side):
        got = call(None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("odd", [0, 1])
def test_two_at_once(dyn, odd):
    first, second = calls(dyn, K=96 + odd, h=160 + odd), calls(dyn, K=64 + odd, h=200 + odd, M=4000, E=7, seed=2)
    want = [[t.clone() for t in c[n](None)] for c in (first, second) for n in NAMES]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [c[n](s) for c, s in ((first, streams[0]), (second, streams[1])) for n in NAMES]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))


@pytest.mark.parametrize("M,K,h,E", [(1, 64, 64, 4), (700, 72, 136, 5), (701, 75, 131, 5), (66000, 256, 512, 4)])
def test_replays_from_a_graph(dyn, M, K, h, E):
    """The step forward and backward as one graph, replayed on new inputs with eager work of the same calls between the replays."""
    g = torch.Generator("cuda").manual_seed(M)
    normal = lambda *shape, std=1.0: (torch.randn(*shape, generator=g, device="cuda") * std).to(BF)
    x, W1, W2, dy = normal(M, K), normal(E, 2, h, K, std=K ** -0.5), normal(E, K, h, std=h ** -0.5), normal(M, K)
    off = torch.linspace(0, M, E + 1, device="cuda").int()
    gamma = torch.ones(K, device="cuda")
    pre, x8, ws = room8(dyn, M, 2, h), room8(dyn, M, K), torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
    out, hidden, dpre, dx = torch.empty(M, h, dtype=BF, device="cuda"), torch.empty(M, h, dtype=BF, device="cuda"), torch.empty(M, 2, h, dtype=BF, device="cuda"), torch.empty_like(x)
    mean, rstd = x.float().mean(1), torch.ones(M, device="cuda")

    def step(pre, x8, out, hidden, dpre, dx):
        dyn.dynb_store8(x, out=x8)
        dyn.moe_gated(x, W1, off, out=out, pre=pre)
        dyn.moe_gated_grad(dy, W2, off, pre, dpre=dpre, hidden=hidden)
        back = dyn.dynb_load8(x8)
        _, dgamma, dbeta = dyn.dynb_layer_norm_backward(dy, x8, gamma, mean, rstd, dx=dx, workspace=ws)
        return [out, pre.q, pre.scale, dpre, hidden, back, dx, dgamma, dbeta]

    fresh = lambda: step(room8(dyn, M, 2, h), room8(dyn, M, K), *(torch.empty_like(t) for t in (out, hidden, dpre, dx)))
    fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step(pre, x8, out, hidden, dpre, dx)
    for rep in range(4):
        x.copy_(normal(M, K))
        dy.copy_(normal(M, K))
        for t in results:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = fresh()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want)), rep
