"""How far a row in 8 bits may be from what was stored, as include/dynbatch.h says it."""
import pytest
import torch

from tests.test_gpu_rows8 import dyn  # noqa: F401

pytestmark = pytest.mark.gpu


def test_how_far_an_element_is_off(dyn):  # noqa: F811
    """By at most half a scale: a / 252 of the block's largest, or 2^-127 where that is below 127 * 2^-126 and the scale is held at 2^-126.  (What x * (1 / s) loses in fp32 comes to
    127 * 2^-23 of a step, 2^-15 of half a scale; a scale is at most 2^-7 above a / 127, so that half of it stays below a / 252 with that.)"""
    g = torch.Generator().manual_seed(4)
    power = torch.arange(-149, 127).repeat_interleave(8)
    x = (torch.rand(len(power), 32, generator=g, dtype=torch.float64) * 2 - 1) * (2.0 ** power.double())[:, None]
    x = torch.cat([x.float(), torch.tensor([[127.0, 126.0]]) * 2.0 ** -126 @ torch.eye(2, 32), torch.full((1, 32), 2.0 ** -127)])
    off = (dyn.dynb_load8(dyn.dynb_store8(x.cuda()), dtype=dyn.DYNB_F32).cpu().double() - x.double()).abs().amax(1)
    a = x.double().abs().amax(1)
    held = a < 127 * 2.0 ** -126
    assert bool((off[~held] <= a[~held] / 252).all()) and bool((off[held] <= 2.0 ** -127).all()) and int(held.sum()) > 100 < int((~held).sum())
    assert float(off[-1]) > float(a[-1]) / 252                               # (the held scale's half is what bounds such a block)
