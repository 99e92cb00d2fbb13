"""Orthogonalised updates over the whole range of norms, eps, steps and sizes of the parts of G, against 64 bits.

A step's products are good to e = 3 (sqrt(l) + 4) u32 of its result, as in the tests at ordinary norms: after T steps the result is off
by at most e (a^T - 1) / (a - 1) of the norm that unamplified directions have.  Where all singular values are small, the whole result
is such a direction, and T e of it bounds the error; the first is larger for every T here.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16
COEF = (3.4445, -4.7750, 2.0315)
U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def il():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_01985_amd as mod
    return mod


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _exact(G, steps, coef=COEF, eps=1e-7):
    a, b, c = coef
    X = G.double()
    tall = X.shape[-2] > X.shape[-1]
    X = X.transpose(-1, -2).contiguous() if tall else X
    X = X / (X.square().sum((-1, -2), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        A = X @ X.transpose(-1, -2).contiguous()
        X = a * X + (b * A + c * A @ A) @ X
    return X.transpose(-1, -2) if tall else X


def _tol(rows, cols, steps, out=F32):
    a = COEF[0]
    return 3 * (math.sqrt(max(rows, cols)) + 4) * U32 * (a ** steps - 1) / (a - 1) + (2.0 ** -8 if out == BF16 else 0.0)


def _far(got, want):
    return float((got.double() - want).norm() / want.norm())


def _of_norm(shape, norm, gen):
    G = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float64)
    return (G * (norm / G.square().sum((-1, -2), keepdim=True).sqrt())).float()


# one workgroup's matrices, general ones, tall ones
@pytest.mark.parametrize("shape", [(64, 220), (220, 60), (600, 700), (1030, 300)])
@pytest.mark.parametrize("norm", [1e-37, 1e-36, 1e-33, 1e38, 3e40])
def test_norms_at_the_ends_of_float32(il, shape, norm):
    """eps = 0: the result does not depend on the norm, though 1 / norm, or the norm itself, is no float32 number."""
    if norm > 1e39 and shape[0] * shape[1] < 300_000:
        pytest.skip("entries would be infinite")
    G = _of_norm((1, *shape), norm, _gen(shape[0]))
    assert bool(torch.isfinite(G).all())
    for steps in (1, 5):
        assert _far(il.ilargi_orthogonalize(G, steps=steps, eps=0.0), _exact(G, steps, eps=0.0)) <= _tol(*shape, steps)


@pytest.mark.parametrize("shape", [(64, 220), (220, 60), (1, 1), (512, 512), (300, 1000), (777, 130), (130, 2500)])
@pytest.mark.parametrize("norm,eps", [(1e-7, 1e-7), (1e-9, 1e-7), (1e-11, 1e-7), (1e-13, 1e-7), (1e-16, 1e-7), (1e-25, 1e-7), (1e-8, 1e-3), (1.0, 1.0),
                                      (1e-3, 1e3), (1e-30, 1.0)])
def test_norms_below_eps(il, shape, norm, eps):
    """X = G / (|G| + eps) is as small as |G| / eps, and the result a^T times that: not less exact for it."""
    G = _of_norm((1, *shape), norm, _gen(shape[0]))
    for steps in (1, 2, 5):
        assert _far(il.ilargi_orthogonalize(G, steps=steps, eps=eps), _exact(G, steps, eps=eps)) <= _tol(*shape, steps)
    assert _far(il.ilargi_orthogonalize(G, eps=eps, out_dtype=BF16), _exact(G, 5, eps=eps)) <= _tol(*shape, 5, BF16)
    assert _far(il.ilargi_orthogonalize(G.bfloat16(), eps=eps, out_dtype=F32), _exact(G.bfloat16(), 5, eps=eps)) <= _tol(*shape, 5)


@pytest.mark.parametrize("shape", [(64, 220), (220, 60), (130, 257), (512, 300)])
def test_a_batch_of_very_different_norms(il, shape):
    """Every matrix by its own norm; a zero one among them, and weights that are updated in place."""
    norms = (1.0, 1e-12, 0.0, 1e-7, 1e-20, 1e5)
    G = torch.cat([_of_norm((1, *shape), v, _gen(q)) for q, v in enumerate(norms)])
    G[2] = 0.0
    out, want = il.ilargi_orthogonalize(G), _exact(G, 5)
    for q, v in enumerate(norms):
        assert bool((out[q] == 0).all()) if v == 0.0 else _far(out[q], want[q]) <= _tol(*shape, 5)
    W = torch.randn(G.shape, generator=_gen(9), device="cuda") * want.float().abs().amax((1, 2), keepdim=True)
    far = 0.99 * W.double() - 0.3 * want
    il.ilargi_orthogonalize(G, out=W, base=W, alpha=-0.3, beta=0.99)
    for q, v in enumerate(norms):
        assert bool((W[q] == 0).all()) if v == 0.0 else _far(W[q], far[q]) <= _tol(*shape, 5)


@pytest.mark.parametrize("coef", [(1.5, -0.5, 0.0), (0.1, 0.0, 0.0), (0.5, 0.25, 0.0)])
def test_other_coefficients_below_eps(il, coef):
    """Iterations that grow slowly, or shrink what they are given: T roundings, none of them amplified beyond the result."""
    for shape in ((60, 220), (300, 200)):
        for norm in (1e-12, 1e-4, 1.0):
            G = _of_norm((1, *shape), norm, _gen(5))
            for steps in (3, 12):
                want = _exact(G, steps, coef)
                assert _far(il.ilargi_orthogonalize(G, steps=steps, coef=coef), want) <= 2 * steps * 3 * (math.sqrt(max(shape)) + 4) * U32


def test_coefficients_that_leave_nothing(il):
    for shape in ((60, 40), (200, 300)):
        assert bool((il.ilargi_orthogonalize(torch.randn(shape, generator=_gen(6), device="cuda"), steps=3, coef=(0.0, 0.0, 0.0)) == 0).all())


def test_negative_eps(il):
    """eps < 0 brings X beyond norm 1: |G| = 1, eps = -0.98 gives X of norm 50."""
    for shape in ((1, 1), (40, 64), (100, 130)):
        G = _of_norm((1, *shape), 1.0, _gen(shape[0]))
        eps = -0.98
        for steps in (1, 3):
            want = _exact(G, steps, (0.1, 0.0, 0.0), eps=float(torch.tensor(eps)))
            assert _far(il.ilargi_orthogonalize(G, steps=steps, coef=(0.1, 0.0, 0.0), eps=eps), want) <= 50 * _tol(*shape, steps)


def _orbit(s, steps):
    """Singular values s_0 .. s_T of one direction, and a bound of the relative error of s_T for errors e in every step: an error of the
    value itself is passed on by p'(s) s / p(s), one of its vectors (all values of a part are equal) as it is."""
    a, b, c = COEF
    values = [s]
    for _ in range(steps):
        x = values[-1]
        values.append(x * (a + b * x * x + c * x ** 4))
    total = 0.0
    for j in range(steps):
        k = 1.0
        for x in values[j:steps]:
            k *= abs((a + 3 * b * x * x + 5 * c * x ** 4) / (a + b * x * x + c * x ** 4))
        total += max(1.0, k)
    return total


@pytest.mark.parametrize("rows,cols", [(32, 64), (64, 400), (96, 256), (512, 300)])
@pytest.mark.parametrize("steps", [7, 8, 10, 15, 20])
@pytest.mark.parametrize("part", [1e-4, 1e-6, 1e-8, 1e-10])
def test_parts_of_very_different_size(il, rows, cols, steps, part):
    """Two parts on rows and columns of their own, each with orthonormal rows, the second scaled far down: they do not mix, and many steps
    bring the second near 1 too.  Each part is good to what float32 products leave of it."""
    gen = _gen(rows + steps)
    G = torch.zeros(rows, cols, device="cuda", dtype=torch.float64)
    r, c = rows // 2, cols // 2
    for q, size in enumerate((1.0, part)):
        m = torch.randn(max(r, c), min(r, c), generator=gen, device="cuda", dtype=torch.float64)
        Q = torch.linalg.qr(m)[0]
        G[q * r: (q + 1) * r, q * c: (q + 1) * c] = (Q if r > c else Q.t()) * size
    G = G.float()
    got, want = il.ilargi_orthogonalize(G, steps=steps), _exact(G, steps)
    e = 3 * (math.sqrt(max(rows, cols)) + 4) * U32
    for q, size in enumerate((1.0, part)):
        rr, cc = slice(q * r, (q + 1) * r), slice(q * c, (q + 1) * c)
        s0 = size / math.sqrt(min(r, c) * (1 + part * part))
        # (the factors of G are orthonormal to a rounding of float32: one more e at the start)
        assert _far(got[rr, cc], want[rr, cc]) <= e * (_orbit(s0, steps) + 1)
    assert bool((got[:r, c:] == 0).all()) and bool((got[r:, :c] == 0).all())


def test_a_base_with_a_side_of_one(il):
    """The stride along a side of length 1 says nothing of the layout: a row, or one matrix, cut from wider weights is read as it lies."""
    wide = torch.randn(8, 96, generator=_gen(3), device="cuda")
    store = torch.empty(8, 96, device="cuda")
    for base, out in ((wide[2:3, :40], torch.empty(1, 40, device="cuda")), (wide[None, :, :40], store.as_strided((1, 8, 40), (7, 96, 1)))):
        G = torch.randn(base.shape, generator=_gen(4), device="cuda")
        want = -0.5 * _exact(G, 5) + base.double()
        assert _far(il.ilargi_orthogonalize(G, out=out, base=base, alpha=-0.5, beta=1.0), want) <= _tol(8, 96, 5)
    with pytest.raises(ValueError):
        il.ilargi_orthogonalize(wide[:, :40], base=wide[:, :40], beta=1.0)      # (out is new, and its rows are shorter)
