"""Layer norm's gradients from rows in 8 bits at widths whose last piece of 16 bytes begins in its neighbour: two lanes then read the same columns, of one wave or of two, and of what they
make the row's end counts once.  In place (dx is dy) both have to have read before either stores."""
import pytest
import torch

from tests.operator_util import U32, gaps_untouched, stored, strided, within
from tests.test_gpu_rows8 import BF, dyn, norm_bounds, normal, to_eight, values  # noqa: F401

pytestmark = pytest.mark.gpu

# The lane with the row's end (a lane has 8 columns in bf16, 4 in fp32, a wave 512 or 256 neighbours): the first of a row's only wave (513, 257), its first with a second piece
# (1025), the last of a wave (511, 2047, 4095, 8191), the first of another wave, whose neighbour is the last of the wave before (2049, 2561, 2305, 4097, 5121, 6913), within one (1000 + 3, 7000 +
# 5); a piece and one more (9, 5), a piece less one (7, 3); sixteen waves (10001, 16383).  Rows: fewer than a launch's workgroups have, and some each.
WIDTHS = [3, 5, 7, 9, 257, 511, 513, 1003, 1025, 2047, 2049, 2051, 2305, 2561, 4095, 4097, 5121, 6913, 7005, 8191, 10001, 16383]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("T,gap", [(37, 0), (37, 3), (2500, 0)])
def test_ends_of_rows_and_in_place(dyn, T, d, dtype, gap):  # noqa: F811
    if T > 1000 and d > 3000:
        T = 1100                                             # (two rows and more a workgroup of 4 waves and of 16)
    x, dy = normal(T, d, torch.float32, T + d) + 0.5, normal(T, d, dtype, T + d + 1, channels=False)
    gamma = 1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(d))
    _, mean, rstd = dyn.dynb_layer_norm(x.cuda(), gamma.cuda(), want_stats=True)
    q, scale = to_eight(x)
    qv, _ = strided(q, gap, torch.int8, gap)
    sv, _ = strided(scale, gap, BF, gap)
    dyv, dyb = strided(dy, gap, dtype, gap)
    kept = dyn.Rows8(qv, sv)
    dx, dgamma, dbeta = dyn.dynb_layer_norm_backward(dyv, kept, gamma.cuda(), mean, rstd)
    (rx, ex), (rg, eg), (rb, eb) = norm_bounds(values(q, scale), dy.double(), gamma.double(), mean.cpu().double()[:, None], rstd.cpu().double()[:, None])
    within(dx, rx, stored(rx, ex, dtype), "dx")
    within(dgamma, rg, eg + U32 * rg.abs(), "dgamma")
    within(dbeta, rb, eb + U32 * rb.abs(), "dbeta")
    got = dyn.dynb_layer_norm_backward(dyv, kept, gamma.cuda(), mean, rstd, dx=dyv)
    assert got[0] is dyv and torch.equal(dyv, dx) and torch.equal(got[1], dgamma) and torch.equal(got[2], dbeta)
    assert gaps_untouched(dyv, dyb, gap)


@pytest.mark.parametrize("d", [9, 513, 2049, 4097, 8191])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_a_row_that_is_no_number_stays_alone(dyn, d, dtype):  # noqa: F811
    """A block, or a gradient, that is NaN at a row's end: that row's dx and those columns of the parameters' gradients, and nothing else"""
    T = 70
    x, dy = normal(T, d, torch.float32, d), normal(T, d, dtype, d + 1, channels=False)
    gamma = torch.ones(d, device="cuda")
    _, mean, rstd = dyn.dynb_layer_norm(x.cuda(), gamma, want_stats=True)
    want = dyn.dynb_layer_norm_backward(dy.cuda(), dyn.dynb_store8(x.cuda()), gamma, mean, rstd)
    x[11, d - 1], dy[23, d - 1] = float("nan"), float("inf")
    dx, dgamma, dbeta = dyn.dynb_layer_norm_backward(dy.cuda(), dyn.dynb_store8(x.cuda()), gamma, mean, rstd)
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[[11, 23]] = False
    block = (d - 1) // 32 * 32
    assert torch.equal(dx[rows], want[0][rows]) and torch.isnan(dx[11]).all() and not torch.isfinite(dx[23]).any()
    assert torch.equal(dgamma[:block], want[1][:block]) and torch.isnan(dgamma[block:]).all()
    assert torch.equal(dbeta[:d - 1], want[2][:d - 1]) and not torch.isfinite(dbeta[d - 1])
