"""Refusals of the operators of models with learned features that need no GPU: they come before any device work."""
import ctypes

import pytest

import paper_2502_01985_amd as il

P, BAD = 1 << 20, 1 << 20 | 8         # addresses that are only looked at


def _embed(table=P, ttype=0, rows=10, cols=8, ld=8, ids=P, n=4, out=P, otype=0, ldo=8):
    return il.lib.ilargi_embed(table, ttype, rows, cols, ld, ids, n, 1.0, 0, out, otype, ldo, None)


def _embed_grad(d=P, otype=0, ldo=8, ids=P, n=4, dt=P, ttype=0, rows=10, cols=8, ldt=8, ws=P, nbytes=1 << 30):
    return il.lib.ilargi_embed_grad(d, otype, ldo, ids, n, 1.0, 0, dt, ttype, rows, cols, ldt, ws, nbytes, None)


@pytest.mark.parametrize("call", [_embed, _embed_grad])
@pytest.mark.parametrize("kwargs,status", [
    (dict(n=-1), il.ERR_SHAPE), (dict(n=1 << 31), il.ERR_SHAPE), (dict(rows=-1), il.ERR_SHAPE), (dict(cols=0), il.ERR_SHAPE),
    (dict(ldo=7), il.ERR_SHAPE), (dict(ttype=2), il.ERR_UNSUPPORTED), (dict(otype=-1), il.ERR_UNSUPPORTED), (dict(ids=None), il.ERR_NULL),
])
def test_embed_refuses(call, kwargs, status):
    assert call(**kwargs) == status
    assert il.ilargi_last_error() != ""


def test_embed_null_and_workspace():
    assert _embed(table=None) == il.ERR_NULL and _embed(out=None) == il.ERR_NULL and _embed(n=0, ids=None, out=None) == il.OK
    assert _embed_grad(dt=None) == il.ERR_NULL and _embed_grad(d=None) == il.ERR_NULL and _embed_grad(ws=None) == il.ERR_NULL
    assert _embed_grad(ws=BAD) == il.ERR_WORKSPACE and _embed_grad(nbytes=16) == il.ERR_WORKSPACE
    assert _embed_grad(rows=0, dt=None, ws=None) == il.OK
    assert il.lib.ilargi_embed_grad_workspace_bytes(4, 10, 8, None) == il.ERR_NULL
    small, large = il.ilargi_embed_grad_workspace_bytes(100, 10, 8), il.ilargi_embed_grad_workspace_bytes(1_000_000, 10, 8)
    assert 0 < small < large and small % 256 == 0


def _layer(n=4, k=6, m=8, type=0, act=1):
    return ctypes.byref(il.LayerStruct(n, k, m, type, act))


def _linear(layer=None, X=P, ldx=6, W=P, ldw=8, res=None, ldr=0, out=P, ldo=8, pre=None, ldp=0, ws=P, nbytes=1 << 40):
    return il.lib.ilargi_linear(layer if layer is not None else _layer(), X, ldx, W, ldw, None, res, ldr, out, ldo, pre, ldp, ws, nbytes, None)


def _linear_grad(layer=None, d=P, ldo=8, pre=P, ldp=8, X=P, ldx=6, W=P, ldw=8, dX=P, lddx=6, dW=P, lddw=8, ws=P, nbytes=1 << 40):
    return il.lib.ilargi_linear_grad(layer if layer is not None else _layer(), d, ldo, pre, ldp, X, ldx, W, ldw, dX, lddx, dW, lddw, None, 0, ws, nbytes, None)


@pytest.mark.parametrize("call", [_linear, _linear_grad])
@pytest.mark.parametrize("layer,status", [
    (dict(n=-1), il.ERR_SHAPE), (dict(k=0), il.ERR_SHAPE), (dict(m=0), il.ERR_SHAPE), (dict(n=1 << 31), il.ERR_SHAPE), (dict(type=5), il.ERR_UNSUPPORTED),
    (dict(act=5), il.ERR_UNSUPPORTED), (dict(act=-1), il.ERR_UNSUPPORTED),
])
def test_layers_that_are_none(call, layer, status):
    assert call(_layer(**layer)) == status
    assert il.lib.ilargi_linear_workspace_bytes(_layer(**layer), None, None) == status


def test_linear_refuses():
    assert il.lib.ilargi_linear_workspace_bytes(None, None, None) == il.ERR_NULL
    for bad in (dict(ldx=5), dict(ldw=7), dict(ldo=7), dict(res=P, ldr=7), dict(pre=P, ldp=7)):
        assert _linear(**bad) == il.ERR_SHAPE
    for bad in (dict(X=None), dict(W=None), dict(out=None)):
        assert _linear(**bad) == il.ERR_NULL
    assert _linear(_layer(n=0), X=None, out=None) == il.OK
    for bad in (dict(ldo=7), dict(ldp=7), dict(ldx=5), dict(ldw=7), dict(lddx=5), dict(lddw=7)):
        assert _linear_grad(**bad) == il.ERR_SHAPE
    for bad in (dict(d=None), dict(pre=None), dict(X=None), dict(W=None), dict(ws=None)):
        assert _linear_grad(**bad) == il.ERR_NULL
    assert _linear_grad(ws=BAD) == il.ERR_WORKSPACE and _linear_grad(nbytes=16) == il.ERR_WORKSPACE


def _ortho(G=P, gtype=0, batch=2, rows=6, cols=4, ldg=4, farg=24, steps=5, beta=0.0, base=None, out=P, otype=0, ldo=4, faro=24, ws=P, nbytes=1 << 40):
    return il.lib.ilargi_orthogonalize(G, gtype, batch, rows, cols, ldg, farg, steps, None, 1e-7, 1.0, beta, base, out, otype, ldo, faro, ws, nbytes, None)


@pytest.mark.parametrize("kwargs,status", [
    (dict(batch=-1), il.ERR_SHAPE), (dict(rows=0), il.ERR_SHAPE), (dict(cols=0), il.ERR_SHAPE), (dict(rows=16385), il.ERR_SHAPE), (dict(steps=0), il.ERR_SHAPE),
    (dict(steps=101), il.ERR_SHAPE), (dict(ldg=3), il.ERR_SHAPE), (dict(ldo=3), il.ERR_SHAPE), (dict(farg=23), il.ERR_SHAPE), (dict(faro=20), il.ERR_SHAPE),
    (dict(gtype=7), il.ERR_UNSUPPORTED), (dict(otype=7), il.ERR_UNSUPPORTED), (dict(G=None), il.ERR_NULL), (dict(out=None), il.ERR_NULL),
    (dict(beta=1.0), il.ERR_NULL), (dict(ws=None), il.ERR_NULL), (dict(ws=BAD), il.ERR_WORKSPACE), (dict(nbytes=100), il.ERR_WORKSPACE),
])
def test_orthogonalize_refuses(kwargs, status):
    assert _ortho(**kwargs) == status
    assert il.ilargi_last_error() != ""


def test_orthogonalize_of_nothing():
    assert _ortho(batch=0, G=None, out=None, ws=None) == il.OK
    assert il.lib.ilargi_orthogonalize_workspace_bytes(1, 4, 4, 0, None) == il.ERR_NULL
