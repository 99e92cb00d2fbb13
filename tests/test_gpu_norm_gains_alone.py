"""Gradients of norms of which no bias and no gate of one row is wanted (a kernel of their own), against 64 bits: every number of threads and pieces of a
row, more rows than the workgroups take in one turn.

Bounds: those of test_gpu_norm.py; sums over rows by the additions that a row's term really goes through: one for every turn of its workgroup and
every row beside it there, then float64.  (With n of them, as that file allows for any order, lost rows would pass.)
"""
import pytest

import test_gpu_norm as base
from test_gpu_exact_sums import COLUMNS, _rows_beside

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

E = base.E
il = base.il
KINDS = [("rms", "rms", "silu"), ("rms", "rms", None), ("none", "rms", "sigmoid"), ("centred", "none", None), ("rms", "centred", "gelu")]


def _sum(bound, terms, n, turns):
    """A sum over n rows with `turns` additions in place of n + 24."""
    want, err = bound
    return want, err - (n + 24 - turns) * E * terms.abs().sum(0)


@pytest.mark.parametrize("dtype,m", [(t, m) for t in COLUMNS for m in COLUMNS[t]])
def test_gains_alone(il, dtype, m):
    gen = base._gen(m)
    beside, groups = _rows_beside(m, dtype)
    n = groups * beside + beside // 2 + 3
    turns = 2 + beside + 4
    mat = lambda scale=1.0, add=0.0: base._matrix(n, m, dtype, gen, 3, 1, scale, add)
    h, x, gates, dr, dy = mat(2.0, 0.5), mat(3.0), mat(), mat(0.01), mat(0.01)
    g1, g2 = ((torch.randn(m, generator=gen, device="cuda") * 0.2 + 1.0).to(dtype) for _ in range(2))
    for first, second, act in KINDS:
        gate, y_in = gates if act is not None else None, dy if second != "none" else None
        args = dict(first=first, gain1=g1, gate=gate, gate_act=act or "none", scale=0.7, x=x, second=second, gain2=g2 if second != "none" else None, eps=base.EPS)
        want = base._oracle((first, second), h, x, gate, g1, None, args["gain2"], None, act or "none", 0.7, dr, y_in)
        got = dict(zip(base.GRADS, il.ilargi_norm_grad(dr, y_in, h, **args)))
        assert got["d_bias1"] is None and got["d_bias2"] is None
        f = base._f(gates.double(), act) if act is not None else 1.0
        n1 = base.Norm(h.double(), torch.zeros_like(h.double()), first)
        want["d_gain1"] = _sum(want["d_gain1"], 0.7 * want["d_x"][0] * f * n1.unit, n, turns)
        if y_in is not None:
            want["d_gain2"] = _sum(want["d_gain2"], dy.double() * base.Norm(*want["r"], second).unit, n, turns)
        for name, t in got.items():
            if t is not None:
                base._close(t, want[name], dtype, (name, first, second, act))
        # the same bits with the biases' sums beside them, which are another kernel's
        more = {k: torch.empty_like(g1) for k in ("d_bias1", *(("d_bias2",) if y_in is not None else ()))}
        for name, t in zip(base.GRADS, il.ilargi_norm_grad(dr, y_in, h, **args, **more)):
            if got[name] is not None:
                assert torch.equal(t, got[name]), name
