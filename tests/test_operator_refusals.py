"""What the operators around the expert layer refuse, through the C ABI: no GPU is needed, every check stands ahead of the first launch."""
import ctypes as ct

import pytest

from paper_1707_02402_amd import binding as b

L, P = b.lib, 4096           # an address that nothing is ever launched with


def code(rc):
    return b.ERRORS.get(rc, rc)


def product(M=4, K=8, N=8, E=2, dtype=1, flags=0, offsets=P, perm=None, k=1, rows=4, x=P, xs=8, W=P, out=P, os_=8):
    return code(L.moe_product(b._ProductShape(M, K, N, E, dtype, flags), b._Groups(offsets, perm, k, rows), x, xs, W, out, os_, None))


def grad_input(M=4, K=8, N=8, E=2, dtype=1, flags=0, offsets=P, perm=None, d=P, ds=8, W=P, act=None, as_=0, out=P, os_=8):
    return code(L.moe_product_grad_input(b._ProductShape(M, K, N, E, dtype, flags), b._Groups(offsets, perm, 1, M), d, ds, W, act, as_, out, os_, None))


def grad_weight(M=4, K=8, N=8, E=2, dtype=1, flags=0, offsets=P, d=P, ds=8, x=P, xs=8, dW=P, gd=0, ws=P, wb=1 << 40):
    return code(L.moe_product_grad_weight(b._ProductShape(M, K, N, E, dtype, flags), b._Groups(offsets, None, 1, M), d, ds, x, xs, dW, gd, ws, wb, None))


@pytest.mark.parametrize("call", [product, grad_input, grad_weight])
@pytest.mark.parametrize("kw,want", [
    (dict(M=-1), "DYNB_E_INVAL"), (dict(K=0), "DYNB_E_INVAL"), (dict(N=0), "DYNB_E_INVAL"), (dict(E=0), "DYNB_E_INVAL"),
    (dict(dtype=0), "DYNB_E_UNSUPPORTED"), (dict(flags=2), "DYNB_E_UNSUPPORTED"), (dict(offsets=None), "DYNB_E_INVAL"), (dict(offsets=P + 2), "DYNB_E_INVAL"),
    (dict(M=(1 << 30) + 1), "DYNB_E_UNSUPPORTED"), (dict(E=(1 << 20) + 1), "DYNB_E_UNSUPPORTED"), (dict(K=(1 << 22) + 1), "DYNB_E_UNSUPPORTED")])
def test_shapes(call, kw, want):
    assert call(**kw) == want


def test_products_arguments():
    for kw in (dict(x=None), dict(W=None), dict(out=None), dict(xs=7), dict(os_=7), dict(x=P + 1), dict(out=P + 1), dict(perm=P, k=0), dict(perm=P, rows=0)):
        assert product(**kw) == "DYNB_E_INVAL", kw
    for kw in (dict(d=None), dict(W=None), dict(out=None), dict(ds=7), dict(os_=7), dict(act=P, as_=7), dict(act=P + 1, as_=8), dict(perm=P)):
        assert grad_input(**kw) == "DYNB_E_INVAL", kw
    for kw in (dict(d=None), dict(x=None), dict(dW=None), dict(ws=None), dict(ds=7), dict(xs=7), dict(dW=P + 2), dict(ws=P + 16)):
        assert grad_weight(**kw) == "DYNB_E_INVAL", kw
    assert grad_weight(gd=5) == "DYNB_E_UNSUPPORTED"
    assert grad_weight(wb=0) == "DYNB_E_WORKSPACE"
    assert product(M=1 << 30, N=1 << 22, os_=1 << 22) == "DYNB_E_UNSUPPORTED"             # more tiles than a launch holds
    assert product(M=0) == 0 and grad_input(M=0) == 0                                     # no work
    assert L.moe_product_grad_weight_workspace_bytes(b._ProductShape(4, 8, 8, 0, 1, 0)) == 0


def test_embeddings():
    def look(T=4, V=5, d=8, dtype=0, tokens=P, table=P, out=P, os_=8):
        return code(L.dynb_embed(b._EmbedShape(T, V, d, dtype, 1.0), tokens, table, out, os_, None))

    def grad(T=4, V=5, d=8, dtype=0, tokens=P, dout=P, ds=8, dt=P, gd=0, ws=P, wb=1 << 40):
        return code(L.dynb_embed_backward(b._EmbedShape(T, V, d, dtype, 1.0), tokens, dout, ds, dt, gd, ws, wb, None))

    for call in (look, grad):
        for kw in (dict(T=-1), dict(V=0), dict(d=0), dict(tokens=None), dict(tokens=P + 2)):
            assert call(**kw) == "DYNB_E_INVAL", kw
        assert call(dtype=3) == "DYNB_E_UNSUPPORTED"
        assert call(T=(1 << 25) + 1) == call(V=(1 << 27) + 1) == call(d=(1 << 28) + 1) == "DYNB_E_UNSUPPORTED"
    for kw in (dict(table=None), dict(out=None), dict(os_=7), dict(table=P + 2), dict(out=P + 1)):
        assert look(**kw) == "DYNB_E_INVAL", kw
    for kw in (dict(dout=None), dict(dt=None), dict(ws=None), dict(ds=7), dict(dout=P + 2), dict(dt=P + 2), dict(ws=P + 8)):
        assert grad(**kw) == "DYNB_E_INVAL", kw
    assert grad(wb=8) == "DYNB_E_WORKSPACE" and grad(gd=2) == "DYNB_E_UNSUPPORTED" and look(T=0) == 0
    assert L.dynb_embed_backward_workspace_bytes(b._EmbedShape(4, 0, 8, 0, 1.0)) == 0


def test_layer_norm():
    def fwd(T=4, d=8, dtype=0, eps=1e-5, x=P, xs=8, gamma=None, beta=None, y=P, ys=8, mean=None, rstd=None):
        return code(L.dynb_layer_norm(b._NormShape(T, d, dtype, eps), x, xs, gamma, beta, y, ys, mean, rstd, None))

    def bwd(T=4, d=8, dtype=0, eps=1e-5, dy=P, ds=8, x=P, xs=8, gamma=None, mean=P, rstd=P, dx=P, dxs=8, dg=P, db=P, ws=P, wb=1 << 40):
        return code(L.dynb_layer_norm_backward(b._NormShape(T, d, dtype, eps), dy, ds, x, xs, gamma, mean, rstd, dx, dxs, dg, db, ws, wb, None))

    for call in (fwd, bwd):
        for kw in (dict(T=-1), dict(d=0), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(xs=7), dict(x=P + 2), dict(gamma=P + 1), dict(mean=P + 2)):
            assert call(**kw) == "DYNB_E_INVAL", kw
        assert call(dtype=2) == call(d=(1 << 28) + 1) == "DYNB_E_UNSUPPORTED"
    for kw in (dict(y=None), dict(ys=7), dict(beta=P + 2), dict(rstd=P + 1)):
        assert fwd(**kw) == "DYNB_E_INVAL", kw
    for kw in (dict(dy=None), dict(mean=None), dict(rstd=None), dict(ws=None), dict(ds=7), dict(dxs=7), dict(dg=P + 2), dict(db=P + 1), dict(ws=P + 64)):
        assert bwd(**kw) == "DYNB_E_INVAL", kw
    assert bwd(wb=8) == "DYNB_E_WORKSPACE" and fwd(T=0) == 0
    assert L.dynb_layer_norm_backward_workspace_bytes(b._NormShape(4, 0, 0, 0.0)) == 0


def test_clipping():
    def clip(tensors=((P, P, 8, 0),), n=None, max_norm=1.0, norm=P, ws=P, wb=1 << 40):
        arr = (b._GradTensor * max(len(tensors), 1))(*tensors)
        return code(L.dynb_clip_gradients(arr, len(tensors) if n is None else n, max_norm, norm, ws, wb, None))

    for kw in (dict(n=-1), dict(norm=None), dict(ws=None), dict(ws=P + 8), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")),
               dict(tensors=((None, P, 8, 0),)), dict(tensors=((P, P, -1, 0),)), dict(tensors=((P + 2, P, 8, 0),)), dict(tensors=((P, P, 8, 0), (P, P + 1, 8, 1)))):
        assert clip(**kw) == "DYNB_E_INVAL", kw
    assert clip(tensors=((P, P, (1 << 42) + 1, 1),)) == "DYNB_E_UNSUPPORTED"
    assert clip(wb=8) == "DYNB_E_WORKSPACE" and clip(tensors=((P, P, 8, 4),)) == "DYNB_E_UNSUPPORTED"
    assert code(L.dynb_clip_gradients(None, 1, 1.0, P, P, 1 << 40, None)) == "DYNB_E_INVAL"
