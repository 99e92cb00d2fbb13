"""Matrices of more than 2^31 elements: norms, layers by group and clipping at their far ends."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16 = torch.bfloat16
E, U = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def il():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_01985_amd as mod
    yield mod
    torch.cuda.empty_cache()


def _large(n, m, gen):
    """n x m of bfloat16: a few rows drawn, the others repeat them."""
    some = torch.randn(512, m, generator=gen, device="cuda").to(BF16)
    return some.repeat((n + 511) // 512, 1)[:n]


def test_norm(il):
    gen = torch.Generator(device="cuda").manual_seed(1)
    n, m = 135_000, 16_384
    h, d = _large(n, m, gen), _large(n, m, gen)
    g = torch.randn(m, generator=gen, device="cuda").to(BF16)
    args = dict(first="rms", gain1=g, second="centred", gain2=g)
    r, y = il.ilargi_norm(h, **args)
    got = il.ilargi_norm_grad(d, d, h, **args)
    for at in (0, n - 600):
        rows = slice(at, at + 600)
        small = il.ilargi_norm(h[rows], **args)
        assert torch.equal(small[0], r[rows]) and torch.equal(small[1], y[rows])
        assert torch.equal(il.ilargi_norm_grad(d[rows], d[rows], h[rows], **args)[0], got[0][rows])


def test_grouped(il):
    gen = torch.Generator(device="cuda").manual_seed(2)
    n, k, m, last = 540_000, 4096, 24, 700
    X, D = _large(n, k, gen), torch.randn(n, m, generator=gen, device="cuda").to(BF16)
    W = (torch.randn(2, k, m, generator=gen, device="cuda") / 64).to(BF16)
    o = torch.tensor([0, n - last, n], dtype=torch.int32, device="cuda")
    out = il.ilargi_grouped_linear(X, W, o)
    dX, dW, db = il.ilargi_grouped_linear_grad(D, X, W, o)
    x, d, w = X[-last:].double(), D[-last:].double(), W[1].double()
    for got, want, size, r in ((out[-last:], x @ w, x.abs() @ w.abs(), k), (dX[-last:], d @ w.t(), d.abs() @ w.t().abs(), m), (dW[1], x.t() @ d, x.t().abs() @ d.abs(), last),
                               (db[1], d.sum(0), d.abs().sum(0), last)):
        err = (r + 4) * E * size
        assert bool(((got.double() - want).abs() <= err + U * (want.abs() + err)).all())
    # and one of the long group's, by its sums of a constant: ones times X
    D.fill_(1.0)
    _, dW, db = il.ilargi_grouped_linear_grad(D, X, W, o, d_X=None)
    want = X[: n - last].sum(0, dtype=torch.float64)
    size = X[: n - last].abs().sum(0, dtype=torch.float64)
    assert bool(((dW[0].double() - want[:, None]).abs() <= (n * E * size + U * want.abs())[:, None] * 1.01).all())
    assert bool(((db[0].double() - (n - last)).abs() <= 1.01 * U * n).all())


def test_clip(il):
    n = 2 ** 31 + 1001
    t = torch.full((n,), 0.5, dtype=BF16, device="cuda")
    t[-3:] = torch.tensor([4.0, -8.0, 2.0], device="cuda")
    want = math.sqrt(0.25 * (n - 3) + 84.0)
    norm = il.ilargi_clip_norm([t], 0.25 * want)
    assert abs(float(norm) - want) <= 1.01 * E * want
    assert t[-3:].tolist() == [1.0, -2.0, 0.5] and bool((t[:-3] == 0.125).all())
    # rows far from each other
    wide = t[: 2 ** 31].view(2, 2 ** 30)[:, :7]
    wide[1] = 3.0
    assert abs(float(il.ilargi_clip_norm([wide], math.inf)) - math.sqrt(7 * (9 + 0.125 ** 2))) <= 1e-5
