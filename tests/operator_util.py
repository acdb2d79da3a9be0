"""Helpers of the tests of the operators around the expert layer: plain forms in 64 bits on the host, and error bounds that follow from the
formats and the lengths of the sums.

U32 = 2^-24 and U16 = 2^-8 are half a unit in the last place of fp32 (24 bits of significand) and bfloat16 (8 bits), relative to the value.  A sum of n products in fp32, in any order and
with any grouping, is off by at most n * 2 U32 * sum |products| (each addition and product rounds once; 2 U32 leaves room for matrix
instructions that round towards zero inside); what is stored in bfloat16 is off by U16 more, relative to itself."""
import numpy as np
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8


def stored(ref, err, dtype):
    """Bound of a stored result whose fp32 value is within `err` of `ref`."""
    u = U16 if dtype == torch.bfloat16 else U32
    return err + u * (ref.abs() + err) + 1e-38


def within(got, ref, bound, what=""):
    got = got.double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), what
    over = (got - ref).abs() - bound
    assert (over <= 0).all(), f"{what}: {int((over > 0).sum())} of {over.numel()} beyond their bound, worst by {float(over.max()):.3e}"


def strided(rows, gap, dtype, offset=0):
    """The host tensor's rows on the device, `gap` elements of 7 between them, the first `offset` elements into the buffer: (view, buffer)."""
    n, w = rows.shape
    buf = torch.full((offset + n * (w + gap) + 1,), 7.0, dtype=dtype, device="cuda")
    view = buf[offset:offset + n * (w + gap)].view(n, w + gap)[:, :w]
    view.copy_(rows)
    return view, buf


def gaps_untouched(view, buf, offset=0):
    n, w = view.shape
    pitch = view.stride(0) if n > 1 else buf.numel() - 1 - offset
    mask = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    mask[offset:offset + n * pitch].view(n, pitch)[:, :w] = False
    return bool((buf[mask] == 7).all())
