"""Centred norms of rows whose entries lie far from 0 and near each other, against 64 bits.

A mean in float32 may be off by S mean|v|, S = (m / 32 + 40) 2^-24 as in test_gpu_norm.py, where the deviations around it are far less.  Here the
deviations c = v - mean are bounded by their own size, and by S^2 of the entries' for what a mean may miss:
    ec = (S + 6 E) (|c| + mean|c| + S mean|v|),
so a constant row of 1000 may come out at 2e-5, not at 4.  The variance is off by S of itself, and by what the deviations' errors give.
"""
import pytest

import test_gpu_norm as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, E, EPS = base.F32, base.BF16, base.E, base.EPS
il = base.il


class Near(base.Norm):
    def __init__(self, v, err, kind):
        super().__init__(v, err, kind)
        if kind != "centred":
            return
        mean = lambda t: t.mean(1, keepdim=True)
        c = v - mean(v)
        missed = self.S * mean(v.abs()) + mean(err)
        ec = err + mean(err) + (self.S + 6 * E) * (c.abs() + mean(c.abs()) + missed)
        self.rel = 2 * self.S + (self.by ** 2) * mean(c.abs() * ec + 0.5 * ec * ec)
        self.err = self.by * ec + self.unit.abs() * self.rel + E * self.unit.abs()


@pytest.fixture(autouse=True)
def bounds(monkeypatch):
    monkeypatch.setattr(base, "Norm", Near)


def _rows(n, m, dtype, gen):
    """Rows of ten kinds in turn, so that constant and ordinary ones share a workgroup and a wavefront."""
    v = torch.randn(n, m, generator=gen, device="cuda")
    for i in range(n):
        kind = i % 10
        if kind < 4:
            v[i] = (100.0, 1000.0, -10_000.0, 7.3)[kind]
        elif kind in (4, 5):                                   # one entry a step away
            v[i] = (1000.0, 96.0)[kind - 4]
            v[i, (7 * i) % m] *= 1.0 + (2.0 ** -23 if dtype == F32 else 2.0 ** -7)
        elif kind == 6:
            v[i] = 10_000.0 + 0.01 * v[i]
        elif kind == 7:
            v[i] = -300.0 + v[i]
    return v.to(dtype)


# every number of threads a row, none of them powers of two
COLUMNS = [3, 13, 30, 61, 220, 333, 700, 1000, 1001, 1800, 3000, 4004, 6001, 7000, 12_000]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", COLUMNS)
def test_rows_near_a_constant(il, dtype, m):
    gen = base._gen(m)
    n = 130
    v, d_r, d_y = _rows(n, m, dtype, gen), (0.01 * torch.randn(n, m, generator=gen, device="cuda")).to(dtype), (0.01 * torch.randn(n, m, generator=gen, device="cuda")).to(dtype)
    vec = lambda scale, add: (torch.randn(m, generator=gen, device="cuda") * scale + add).to(dtype)
    gain, bias = vec(0.2, 1.0), vec(0.1, 0.0)
    for first, second, g1, b1, g2, b2 in (("centred", "none", gain, None, None, None), ("centred", "none", gain, bias, None, None), ("none", "centred", None, None, gain, bias)):
        args = dict(first=first, second=second, gain1=g1, bias1=b1, gain2=g2, bias2=b2, eps=EPS)
        dy = d_y if second != "none" else None
        want = base._oracle((first, second), v, None, None, g1, b1, g2, b2, "none", 1.0, d_r, dy)
        r, y = il.ilargi_norm(v, **args)
        base._close(r, want["r"], dtype, ("r", first))
        if y is not None:
            base._close(y, want["y"], dtype, ("y", first))
        back = dict(zip(base.GRADS, il.ilargi_norm_grad(d_r, dy, v, d_x=torch.empty_like(v), **args)))
        for name, t in back.items():
            if t is not None:
                base._close(t, want[name], dtype, (name, first))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", [220, 1000, 5000])
def test_constant_rows_are_their_bias(il, dtype, m):
    """Nothing is left of a constant row but what is added to it: ec by with c = 0, three times (S + 6 E) S |v| / sqrt(eps)."""
    S = (m / 32 + 40) * E
    for value in (1.0, 1000.0, -10_000.0):
        h = torch.full((37, m), value, dtype=dtype, device="cuda")
        r, _ = il.ilargi_norm(h, first="centred")
        most = 3 * (S + 6 * E) * S * abs(value) / EPS ** 0.5
        assert float(r.abs().max()) <= most, value
        _, y = il.ilargi_norm(torch.zeros_like(h), first="none", x=h, second="centred")
        assert float(y.abs().max()) <= most, value


def test_variances_beyond_float32_are_what_float32_gives(il):
    """Squares that no float32 holds make a variance of infinity, and zeros."""
    for m in (40, 700, 1000, 5000):
        h = torch.randn(9, m, generator=base._gen(m), device="cuda") * 1e30 + 3e30
        r, y = il.ilargi_norm(h, first="centred", x=torch.ones_like(h), second="rms")
        assert bool((r == 1).all()) and bool(torch.isfinite(y).all())
