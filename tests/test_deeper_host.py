"""Refusals of the norms, the layers by group and the clipping that need no GPU: they come before any device work."""
import ctypes
import math

import pytest

import paper_2502_01985_amd as il

P, BAD = 1 << 20, 1 << 20 | 8         # addresses that are only looked at


def _block(n=4, m=8, type=0, first=1, second=1, act=0, gate_rows=0, eps=1e-6, h=P, gate=None, x=None, gain2=None, bias2=None, ldh=8, ldg=0, ldx=0):
    return ctypes.byref(il.NormStruct(n, m, type, first, second, act, gate_rows, 1.0, eps, h, None, None, gate, x, gain2, bias2, ldh, ldg, ldx))


def _norm(block=None, r=P, ldr=8, y=P, ldy=8):
    return il.lib.ilargi_norm(block if block is not None else _block(), r, ldr, y, ldy, None)


def _norm_grad(block=None, dr=P, lddr=8, dy=P, lddy=8, ws=P, nbytes=1 << 40, grads=True, **out):
    names = [f[0] for f in il.NormGradsStruct._fields_]
    g = il.NormGradsStruct(**{k: out.get(k, 8 if k.startswith("ld") else None) for k in names})
    return il.lib.ilargi_norm_grad(block if block is not None else _block(), dr, lddr, dy, lddy, ctypes.byref(g) if grads else None, 0, ws, nbytes, None)


@pytest.mark.parametrize("call", [_norm, _norm_grad])
@pytest.mark.parametrize("kwargs,status", [
    (dict(n=-1), il.ERR_SHAPE), (dict(n=1 << 31), il.ERR_SHAPE), (dict(m=0), il.ERR_SHAPE), (dict(m=16385, ldh=16385), il.ERR_SHAPE), (dict(ldh=7), il.ERR_SHAPE),
    (dict(x=P, ldx=7), il.ERR_SHAPE), (dict(gate=P, gate_rows=1, ldg=7), il.ERR_SHAPE), (dict(eps=-1.0), il.ERR_SHAPE), (dict(eps=math.nan), il.ERR_SHAPE),
    (dict(type=2), il.ERR_UNSUPPORTED), (dict(first=3), il.ERR_UNSUPPORTED), (dict(second=-1), il.ERR_UNSUPPORTED), (dict(act=5), il.ERR_UNSUPPORTED),
    (dict(gate_rows=2), il.ERR_UNSUPPORTED), (dict(second=0, gain2=P), il.ERR_UNSUPPORTED), (dict(second=0, bias2=P), il.ERR_UNSUPPORTED), (dict(h=None), il.ERR_NULL),
])
def test_norm_refuses(call, kwargs, status):
    assert call(_block(**kwargs)) == status
    assert il.ilargi_last_error() != ""


def test_norm_outputs_and_workspace():
    assert il.lib.ilargi_norm(None, P, 8, P, 8, None) == il.ERR_NULL
    assert _norm(ldr=7) == il.ERR_SHAPE and _norm(ldy=7) == il.ERR_SHAPE and _norm(_block(second=0)) == il.ERR_UNSUPPORTED
    assert _norm(_block(n=0, h=None)) == il.OK and _norm(r=None, y=None) == il.OK
    assert _norm_grad(grads=False) == il.ERR_NULL
    for bad in (dict(lddr=7), dict(lddy=7), dict(d_h=P, ld_h=7), dict(d_x=P, ld_x=7)):
        assert _norm_grad(**bad) == il.ERR_SHAPE
    assert _norm_grad(_block(gate=P, gate_rows=1, ldg=8), d_gate=P, ld_gate=7) == il.ERR_SHAPE
    assert _norm_grad(d_gate=P) == il.ERR_UNSUPPORTED
    assert _norm_grad(_block(second=0)) == il.ERR_UNSUPPORTED and _norm_grad(_block(second=0), dy=None, d_gain2=P) == il.ERR_UNSUPPORTED
    for out in ("d_gain1", "d_bias1", "d_gain2", "d_bias2"):
        assert _norm_grad(ws=None, **{out: P}) == il.ERR_NULL and _norm_grad(ws=BAD, **{out: P}) == il.ERR_WORKSPACE
        assert _norm_grad(nbytes=16, **{out: P}) == il.ERR_WORKSPACE
    assert il.lib.ilargi_norm_grad_workspace_bytes(4, 8, 0, None) == il.ERR_NULL
    size = ctypes.c_size_t()
    assert il.lib.ilargi_norm_grad_workspace_bytes(4, 0, 0, ctypes.byref(size)) == il.ERR_SHAPE
    assert il.lib.ilargi_norm_grad_workspace_bytes(4, 8, 2, ctypes.byref(size)) == il.ERR_UNSUPPORTED


def _groups(groups=3, n=4, k=6, m=8, type=0, act=1):
    return ctypes.byref(il.GroupsStruct(groups, n, k, m, type, act))


def _grouped(y=None, offsets=P, X=P, ldx=6, W=P, ldw=8, farw=48, bias=None, ldb=0, res=None, ldr=0, out=P, ldo=8, pre=None, ldp=0, ws=P, nbytes=1 << 40):
    return il.lib.ilargi_grouped_linear(y if y is not None else _groups(), offsets, X, ldx, W, ldw, farw, bias, ldb, res, ldr, out, ldo, pre, ldp, ws, nbytes, None)


def _grouped_grad(y=None, offsets=P, d=P, ldo=8, pre=P, ldp=8, X=P, ldx=6, W=P, ldw=8, farw=48, dX=P, lddx=6, dW=P, lddw=8, fardw=48, db=P, lddb=8, ws=P, nbytes=1 << 40):
    return il.lib.ilargi_grouped_linear_grad(y if y is not None else _groups(), offsets, d, ldo, pre, ldp, X, ldx, W, ldw, farw, dX, lddx, dW, lddw, fardw, db, lddb, 0,
                                             ws, nbytes, None)


@pytest.mark.parametrize("call", [_grouped, _grouped_grad])
@pytest.mark.parametrize("layer,status", [
    (dict(groups=-1), il.ERR_SHAPE), (dict(groups=65536), il.ERR_SHAPE), (dict(n=-1), il.ERR_SHAPE), (dict(n=1 << 31), il.ERR_SHAPE), (dict(k=0), il.ERR_SHAPE),
    (dict(m=0), il.ERR_SHAPE), (dict(k=1 << 31), il.ERR_SHAPE), (dict(n=(1 << 31) - 1, m=1 << 20), il.ERR_SHAPE), (dict(type=5), il.ERR_UNSUPPORTED),
    (dict(act=5), il.ERR_UNSUPPORTED), (dict(act=-1), il.ERR_UNSUPPORTED),
])
def test_groups_that_are_none(call, layer, status):
    assert call(_groups(**layer)) == status
    assert il.lib.ilargi_grouped_linear_workspace_bytes(_groups(**layer), None, None) == status


def test_grouped_refuses():
    assert il.lib.ilargi_grouped_linear_workspace_bytes(None, None, None) == il.ERR_NULL
    for bad in (dict(ldx=5), dict(ldw=7), dict(farw=47), dict(ldo=7), dict(bias=P, ldb=7), dict(res=P, ldr=7), dict(pre=P, ldp=7)):
        assert _grouped(**bad) == il.ERR_SHAPE
    for bad in (dict(X=None), dict(W=None), dict(out=None), dict(offsets=None), dict(ws=None)):
        assert _grouped(**bad) == il.ERR_NULL
    assert _grouped(ws=BAD) == il.ERR_WORKSPACE and _grouped(nbytes=16) == il.ERR_WORKSPACE
    assert _grouped(_groups(n=0), X=None, out=None) == il.OK and _grouped(_groups(groups=0), W=None) == il.OK
    for bad in (dict(ldo=7), dict(ldp=7), dict(ldx=5), dict(ldw=7), dict(farw=40), dict(lddx=5), dict(lddw=7), dict(fardw=40), dict(lddb=7)):
        assert _grouped_grad(**bad) == il.ERR_SHAPE
    for bad in (dict(d=None), dict(pre=None), dict(X=None), dict(W=None), dict(ws=None), dict(offsets=None)):
        assert _grouped_grad(**bad) == il.ERR_NULL
    assert _grouped_grad(ws=BAD) == il.ERR_WORKSPACE and _grouped_grad(nbytes=16) == il.ERR_WORKSPACE
    assert _grouped_grad(dX=None, dW=None, db=None) == il.OK and _grouped_grad(_groups(groups=0), offsets=None) == il.OK


def test_grouped_workspaces():
    """The gradient's holds a copy of g; the forward call's holds shares of k, which few rows have and many do not."""
    small, large = (il.ilargi_grouped_linear_workspace_bytes(8, n, 64, 96, il.torch.bfloat16) for n in (100, 100_000))
    assert all(v > 0 and v % 256 == 0 for v in (*small, *large))
    assert small[1] < large[1] and large[1] >= 100_000 * 96 * 2


def _tensors(*entries):
    out = (il.TensorStruct * max(len(entries), 1))()
    for q, e in enumerate(entries):
        out[q] = il.TensorStruct(*e)
    return out


def _clip(entries, max_norm=1.0, ws=P, nbytes=1 << 40, count=None):
    """Refusals only: a call that is none would run."""
    return il.lib.ilargi_clip_norm(_tensors(*entries), len(entries) if count is None else count, max_norm, None, ws, nbytes, None)


@pytest.mark.parametrize("entry,status", [
    ((P, P, -1, 8, 8, 8, 0), il.ERR_SHAPE), ((P, P, 4, -1, 8, 8, 0), il.ERR_SHAPE), ((P, P, 4, 8, 7, 8, 0), il.ERR_SHAPE), ((P, P, 4, 8, 8, 7, 0), il.ERR_SHAPE),
    ((P, P, 4, 8, 8, 9, 0), il.ERR_SHAPE), ((None, P, 4, 8, 8, 8, 0), il.ERR_NULL), ((P, P, 1 << 30, 8, 1 << 20, 1 << 20, 0), il.ERR_SHAPE), ((P, None, (1 << 31) - 1, 1 << 40, 1 << 40, 0, 0), il.ERR_SHAPE), ((P, P, 4, 8, 8, 8, 2), il.ERR_UNSUPPORTED),
    ((P, P + 4, 4, 8, 8, 8, 0), il.ERR_SHAPE), ((P, P + 32, 4, 8, 8, 8, 0), il.ERR_SHAPE),
])
def test_clip_refuses_tensors(entry, status):
    assert _clip([entry]) == status
    assert il.ilargi_last_error() != ""


def test_clip_refuses():
    one = (P, P, 4, 8, 8, 8, 0)
    assert _clip([one], count=-1) == il.ERR_SHAPE and _clip([one], count=65536) == il.ERR_SHAPE
    assert il.lib.ilargi_clip_norm(None, 1, 1.0, None, P, 1 << 40, None) == il.ERR_NULL
    assert _clip([one], max_norm=-1.0) == il.ERR_SHAPE and _clip([one], max_norm=math.nan) == il.ERR_SHAPE
    assert _clip([one], ws=None) == il.ERR_NULL and _clip([one], ws=BAD) == il.ERR_WORKSPACE and _clip([one], nbytes=4) == il.ERR_WORKSPACE
    assert il.lib.ilargi_clip_norm_workspace_bytes(_tensors(one), 1, None) == il.ERR_NULL


def test_clip_refuses_outputs_that_overlap():
    # (a workspace of none refuses what the overlaps let pass: nothing runs here)
    ok = lambda *e: _clip(e, ws=None) == il.ERR_NULL
    far = 1 << 30
    assert ok((P, P, 4, 8, 8, 8, 0), (P + 128, P + 128, 4, 8, 8, 8, 0))
    assert not ok((P, P, 4, 8, 8, 8, 0), (P, P, 4, 8, 8, 8, 0))                       # the same one twice, in place
    assert ok((P, None, 4, 8, 8, 8, 0), (P, None, 4, 8, 8, 8, 0))                     # ... only counted twice
    assert ok((P, far, 4, 8, 8, 8, 0), (P, far + 128, 4, 8, 8, 8, 0))                 # ... into places of their own
    assert not ok((P, far, 4, 8, 8, 8, 0), (P, far + 124, 4, 8, 8, 8, 0))
    assert not ok((P, P, 4, 8, 8, 8, 0), (P + 64, None, 4, 8, 8, 8, 0))               # read behind another's back
    # column blocks of one matrix of 16 columns
    assert ok((P, P, 4, 8, 16, 16, 0), (P + 32, P + 32, 4, 8, 16, 16, 0))
    assert ok((P + 32, P + 32, 4, 8, 16, 16, 0), (P, P, 5, 8, 16, 16, 0), (P + 64, P + 64, 1, 8, 8, 8, 0)) is False
    assert not ok((P, P, 4, 8, 16, 16, 0), (P + 28, P + 28, 4, 8, 16, 16, 0))
    assert not ok((P, P, 4, 8, 16, 16, 0), (P + 32, P + 32, 4, 9, 16, 16, 0))
    assert not ok((P, P, 4, 8, 16, 16, 0), (P + 32, P + 32, 4, 8, 17, 17, 0))
    assert not ok((P, P, 4, 8, 16, 16, 0), (P + 32, P + 32, 4, 8, 16, 16, 1))
    assert ok((P, P, 4, 8, 16, 16, 0), (P + 32 + 64, P + 32 + 64, 1, 8, 8, 8, 0))     # a vector between its rows


def test_activations_and_norms_by_name():
    with pytest.raises(ValueError):
        il._norm_code("layer")
    assert [il._norm_code(k) for k in ("none", "rms", "centred")] == [0, 1, 2]


def test_python_refuses_tensors_that_are_on_no_device():
    t = il.torch.zeros(4, 8)
    for call in (lambda: il.ilargi_norm(t), lambda: il.TensorList([t]), lambda: il.ilargi_grouped_linear(t, t.unsqueeze(0), t)):
        with pytest.raises(TypeError):
            call()
