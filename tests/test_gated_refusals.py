"""What the gated layer and the rows in 8 bits refuse, through the C ABI: no GPU is needed, every check stands ahead of the first launch."""
import ctypes as ct

import pytest

from paper_1707_02402_amd import binding as b
from tests.test_operator_refusals import L, P, code


def pre_of(rows=P, stride=16, scale=P, scale_stride=2, dtype=1):
    return b._GatedPre(rows, stride, scale, scale_stride, dtype)


def gated(M=4, K=8, h=8, E=2, dtype=1, flags=0, offsets=P, perm=None, k=1, rows=4, x=P, xs=8, W=P, out=P, os_=8, pre=None):
    return code(L.moe_gated(b._GatedShape(M, K, h, E, dtype, flags), b._Groups(offsets, perm, k, rows), x, xs, W, out, os_, pre, None))


def grad(M=4, K=8, h=8, E=2, dtype=1, flags=0, offsets=P, perm=None, d=P, ds=8, W=P, pre=pre_of(), dp=P, dps=16, hid=None, hs=0):
    return code(L.moe_gated_grad(b._GatedShape(M, K, h, E, dtype, flags), b._Groups(offsets, perm, 1, M), d, ds, W, pre, dp, dps, hid, hs, None))


@pytest.mark.parametrize("call", [gated, grad])
@pytest.mark.parametrize("kw,want", [
    (dict(M=-1), "DYNB_E_INVAL"), (dict(K=0), "DYNB_E_INVAL"), (dict(h=0), "DYNB_E_INVAL"), (dict(E=0), "DYNB_E_INVAL"), (dict(dtype=0), "DYNB_E_UNSUPPORTED"),
    (dict(flags=2), "DYNB_E_UNSUPPORTED"), (dict(offsets=None), "DYNB_E_INVAL"), (dict(offsets=P + 2), "DYNB_E_INVAL"), (dict(M=(1 << 30) + 1), "DYNB_E_UNSUPPORTED"),
    (dict(E=(1 << 20) + 1), "DYNB_E_UNSUPPORTED"), (dict(K=(1 << 22) + 1), "DYNB_E_UNSUPPORTED"), (dict(h=(1 << 21) + 1), "DYNB_E_UNSUPPORTED"),
    (dict(W=None), "DYNB_E_INVAL"), (dict(W=P + 1), "DYNB_E_INVAL"), (dict(pre=pre_of(rows=None)), "DYNB_E_INVAL"), (dict(pre=pre_of(stride=15)), "DYNB_E_INVAL"),
    (dict(pre=pre_of(dtype=0)), "DYNB_E_UNSUPPORTED"), (dict(pre=pre_of(dtype=2, scale=None)), "DYNB_E_INVAL"), (dict(pre=pre_of(dtype=2, scale_stride=1)), "DYNB_E_INVAL"),
    (dict(pre=pre_of(rows=P + 1)), "DYNB_E_INVAL"), (dict(pre=pre_of(dtype=2, scale=P + 1)), "DYNB_E_INVAL")])
def test_shapes(call, kw, want):
    assert call(**kw) == want


def test_arguments():
    for kw in (dict(x=None), dict(out=None), dict(xs=7), dict(os_=7), dict(x=P + 1), dict(out=P + 1), dict(perm=P, k=0), dict(perm=P, rows=0)):
        assert gated(**kw) == "DYNB_E_INVAL", kw
    for kw in (dict(d=None), dict(dp=None), dict(pre=None), dict(ds=7), dict(dps=15), dict(hid=P, hs=7), dict(hid=P + 1, hs=8), dict(d=P + 1), dict(dp=P + 1), dict(perm=P)):
        assert grad(**kw) == "DYNB_E_INVAL", kw
    assert gated(M=1 << 30, h=1 << 21, os_=1 << 21) == "DYNB_E_UNSUPPORTED"               # more tiles than a launch holds
    assert gated(M=0) == 0 and grad(M=0) == 0 and gated(M=0, x=None, out=None) == 0       # no work
    assert code(L.moe_gated(None, b._Groups(P, None, 1, 4), P, 8, P, P, 8, None, None)) == "DYNB_E_INVAL"


def test_rows_in_eight_bits():
    def rows(q=P, q_stride=40, scale=P, scale_stride=2):
        return b._Rows8(q, q_stride, scale, scale_stride)

    def store(T=4, d=40, dtype=1, x=P, xs=40, r=rows()):
        return code(L.dynb_store8(b._Rows8Shape(T, d, dtype), x, xs, r, None))

    def load(T=4, d=40, dtype=1, x=P, xs=40, r=rows()):
        return code(L.dynb_load8(b._Rows8Shape(T, d, dtype), r, x, xs, None))

    def norm(T=4, d=40, dtype=1, x=P, xs=40, r=rows(), mean=P, ws=P, wb=1 << 40):
        return code(L.dynb_layer_norm_backward8(b._NormShape(T, d, dtype, 1e-5), x, xs, r, None, mean, P, P, 40, P, P, ws, wb, None))

    for call in (store, load, norm):
        for kw in (dict(T=-1), dict(d=0), dict(x=None), dict(xs=39), dict(x=P + 1), dict(dtype=0, x=P + 2), dict(r=None), dict(r=rows(q=None)), dict(r=rows(scale=None)),
                   dict(r=rows(q_stride=39)), dict(r=rows(scale_stride=1)), dict(r=rows(scale=P + 1))):
            assert call(**kw) == "DYNB_E_INVAL", (call, kw)
        assert call(dtype=2) == call(d=(1 << 28) + 1) == "DYNB_E_UNSUPPORTED"
    assert store(T=0) == 0 and load(T=0) == 0
    assert norm(mean=None) == norm(ws=None) == norm(ws=P + 64) == "DYNB_E_INVAL" and norm(wb=8) == "DYNB_E_WORKSPACE"
