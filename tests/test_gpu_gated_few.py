"""moe_gated for few rows with nothing kept (tokens that are being answered): sums shared among waves, groups of one to 16 rows, against the formulas in 64 bits."""
import pytest
import torch

from tests.operator_util import stored, within
from tests.test_gpu_gated import BF, bf, code, dev, dyn, forward_ref, layout  # noqa: F401

pytestmark = pytest.mark.gpu


# rows, channels, hidden features, experts: channels below one wave's, ending inside a wave's 64, a whole turn of all waves (2048, 1024 with two blocks) and more; features around blocks
# of 8 and 16; one group, rows fewer and more than groups, more groups than are counted (2048); enough blocks for two a workgroup (4096 features) and for the tiles (16 rows of 64 groups)
@pytest.mark.parametrize("M,K,h,E,loads", [
    (1, 8, 1, 1, "last"), (1, 64, 8, 1, "last"), (1, 72, 9, 3, "last"), (2, 200, 333, 4, "ones"), (3, 520, 7, 300, "skew"), (4, 2048, 40, 2, "skew"), (5, 2056, 17, 5, "tail"),
    (7, 1000, 1000, 1, "last"), (8, 4104, 65, 8, "skew"), (9, 328, 129, 2, "first"), (15, 512, 1024, 1, "last"), (16, 136, 250, 3, "skew"), (16, 1032, 4100, 1, "last"),
    (16, 64, 96, 64, "ones"), (16, 1024, 4096, 3, "skew"), (2, 4096, 4096, 64, "ones"), (12, 96, 200, 2500, "skew"), (4, 128, 2040, 40, "tail")])
@pytest.mark.parametrize("gate,gathered", [("silu", False), ("gelu", True)])
def test_few_rows(dyn, M, K, h, E, loads, gate, gathered):  # noqa: F811
    g, off, off_d = layout(M, E, loads, M * 5 + K + h)
    k = 2 if gathered else 1
    n_rows = (M + k - 1) // k if gathered else M
    x, W = bf(g, n_rows, K), torch.randn(E, 2, h, K, generator=g).mul_(K ** -0.5).to(BF)
    perm = torch.randperm(M, generator=g).int() if gathered else None
    rows = x[perm.long() // k] if gathered else x
    live = [e for e in range(E) if off[e + 1] > off[e]]
    few = [0] + [int(off[e + 1]) for e in live]
    _, _, ref, bound = forward_ref(x, W[live].double() if live else W[:0].double(), few, rows, gate)
    whole = torch.full((M, h + 5), 7.0, dtype=BF, device="cuda")
    for out in (torch.full((M, h), float("nan"), dtype=BF, device="cuda"), whole[:, 3:3 + h]):
        args = dict(perm=perm.cuda() if gathered else None, k=k, gate=code(dyn, gate))
        dyn.moe_gated(dev(x), W.cuda(), off_d, out=out, **args)
        within(out, ref, stored(ref, bound, BF))
        assert torch.equal(dyn.moe_gated(dev(x), W.cuda(), off_d, **args), out)
    assert bool((whole[:, :3] == 7).all()) and bool((whole[:, 3 + h:] == 7).all())


def test_a_row_that_is_no_number_stays_alone(dyn):  # noqa: F811
    """16 rows are one product's columns: an infinity or a NaN in one of them, or in a feature's weights, is in no other's sum"""
    M, K, h = 11, 1096, 90
    g, _, off = layout(M, 1, "last", 3)
    x, W = bf(g, M, K).to(BF).cuda(), bf(g, 1, 2, h, K, std=K ** -0.5).to(BF).cuda()
    want = dyn.moe_gated(x, W, off)
    x[4, K - 1], x[7, 0], W[0, 0, 33, 500], W[0, 1, 89, K - 1] = float("nan"), float("inf"), float("nan"), float("nan")
    got = dyn.moe_gated(x, W, off)
    whole = torch.ones(M, h, dtype=torch.bool, device="cuda")
    whole[[4, 7]] = False
    whole[:, [33, 89]] = False
    assert torch.equal(got[whole], want[whole]) and bool(got[4].isnan().all()) and bool(got[:, [33, 89]].isnan().all()) and not bool(got[7].isfinite().any())


def test_replays_of_a_step_of_tokens(dyn):  # noqa: F811
    """A captured call reads what its buffers hold at every replay: other tokens, other loads, rows of no group among them"""
    M, K, h, E = 6, 264, 100, 9
    g = torch.Generator().manual_seed(1)
    W = bf(g, E, 2, h, K, std=K ** -0.5).to(BF).cuda()
    x, off, perm = torch.zeros(M, K, dtype=BF, device="cuda"), torch.zeros(E + 1, dtype=torch.int32, device="cuda"), torch.zeros(M, dtype=torch.int32, device="cuda")
    out = torch.empty(M, h, dtype=BF, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        dyn.moe_gated(x, W, off, perm=perm, out=out)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dyn.moe_gated(x, W, off, perm=perm, out=out)
    for n in range(5):
        rows = torch.bincount(torch.randint(E, (M - n % 2 * 2,), generator=g), minlength=E)
        x.copy_(bf(g, M, K))
        perm.copy_(torch.randperm(M, generator=g).int())
        off.copy_(torch.cat([torch.zeros(1, dtype=torch.long), rows.cumsum(0)]).int())
        out.fill_(float("nan"))
        graph.replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(dyn.moe_gated(x, W, off, perm=perm), got)
        assert bool((got[int(off[E]):] == 0).all()) and bool(got.isfinite().all())
