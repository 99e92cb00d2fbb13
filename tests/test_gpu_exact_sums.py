"""Sums over many rows whose values are whole numbers: the results have to be equal, so that no row, chunk or part of rows can be missing.

Every term is a whole number of at most 16 other than 0, and the second half of the rows (of every group) takes back what the first half adds,
but for a few rows: sums on the way stay below 2^24, where float32 is exact, and totals below 2^8, where bfloat16 is.  A row that is missing or counted
twice changes every column, one of a half with it the whole chunk or part.  The norms' sums of what a norm has made go over rows of one size, +-c:
each unit value is +-rho with one rho, off 1 by at most 8 E (the mean, eps 1e-6 below c^2 E, the root, the products), so a total T is off by
8 E |T| and the roundings of its additions, 2^-24 of the largest sum on the way for each of them: below 0.1, where a row is 1 at least.
"""
import pytest

import test_gpu_norm as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16
il = base.il


def _whole(shape, gen, most=2):
    """Whole numbers from -most to most, none of them 0."""
    v = torch.randint(1, most + 1, shape, generator=gen, device="cuda").float()
    return torch.where(torch.rand(shape, generator=gen, device="cuda") < 0.5, -v, v)


def _halves(same, opposite, gen, few):
    """The second half of the rows repeats the first of `same` and has the negative of `opposite`, but for `few` rows of those."""
    n = same.shape[0]
    half = n // 2
    same[n - half:] = same[:half]
    opposite[n - half:] = -opposite[:half]
    if n > 0:
        some = torch.randint(0, n, (few,), generator=gen, device="cuda")
        opposite[some] = -opposite[some]


def _seen(terms):
    """No row's terms are 0: its loss shows in every column."""
    assert bool((terms != 0).all())


def _rows_beside(m, dtype):
    """Rows of a workgroup and the most workgroups of a gradient, by the pieces of 16 bytes of a row."""
    pieces = -(-m // (4 if dtype == F32 else 8))
    for width in (4, 8, 16, 64, 128, 256):
        if pieces <= width:
            return 256 // width, 768
    return 1, 256


# shorter than a piece; then odd, whole and full rows of every number of threads and pieces
COLUMNS = {F32: [3, 13, 12, 16, 30, 28, 32, 61, 60, 64, 255, 220, 256, 511, 508, 512, 1001, 1000, 1024, 2047, 2000, 2048, 4001, 4000, 4096, 6001, 6000, 8192, 9001, 12_000, 16_384],
           BF16: [7, 30, 24, 32, 61, 56, 64, 127, 120, 128, 511, 504, 512, 1001, 1000, 1024, 2047, 2000, 2048, 4001, 4000, 4096, 6001, 6000, 8192, 9001, 12_000, 16_384]}


@pytest.mark.parametrize("dtype,m", [(t, m) for t in COLUMNS for m in COLUMNS[t]])
def test_sums_of_a_norm_over_rows(il, dtype, m):
    gen = base._gen(m)
    beside, groups = _rows_beside(m, dtype)
    n = 2 * groups * beside + beside // 2 + 7           # two turns of every workgroup, and a part of a third
    h, gate, dr, dy, c = _whole((n, m), gen), _whole((n, m), gen), _whole((n, m), gen), _whole((n, m), gen), _whole((n, m), gen, 1) * 4096.0
    row = _whole((m,), gen)
    _halves(h, dr, gen, 2)
    gate[n - n // 2:] = gate[: n // 2]
    _halves(c, dy, gen, 2)
    new = lambda: torch.full((m,), float("nan"), dtype=dtype, device="cuda")
    H, G, DR, DY, C, R = (t.to(dtype) for t in (h, gate, dr, dy, c, row))
    D = torch.float64
    equal = lambda got, want: torch.equal(got.double(), want)
    # gains alone, gates of their own
    t = 2.0 * dr.to(D) * gate.to(D)
    _seen(t * h.to(D))
    got = il.ilargi_norm_grad(DR, None, H, first="none", gate=G, scale=2.0, d_h=None, d_x=None, d_gate=None, d_gain1=new())[3]
    want = (t * h.to(D)).sum(0)
    assert float(want.abs().max()) <= 128 and equal(got, want)
    old = torch.ones_like(got)
    il.ilargi_norm_grad(DR, None, H, first="none", gate=G, scale=2.0, d_h=None, d_x=None, d_gate=None, d_gain1=old, accumulate=True)
    assert equal(old, want + 1)
    # with the biases' too
    got = il.ilargi_norm_grad(DR, None, H, first="none", gate=G, scale=2.0, d_h=None, d_x=None, d_gate=None, d_gain1=new(), d_bias1=new())
    assert equal(got[3], want) and equal(got[4], t.sum(0))
    # one gate for all rows
    t = dr.to(D) * row.to(D)
    got = il.ilargi_norm_grad(DR, None, H, first="none", gate=R, d_h=None, d_x=None, d_gate=new(), d_gain1=new(), d_bias1=new())
    for a, b in zip(got[2:5], ((h.to(D) * dr.to(D)).sum(0), (t * h.to(D)).sum(0), t.sum(0))):
        assert equal(a, b)
    # the second norm's, of rows of one size: alone, and with all others
    near = lambda got, want: bool(((got.double() - want).abs() <= 0.1).all())
    want = (dy.to(D) * c.to(D) / 4096.0).sum(0)
    _seen(dy * c)
    got = il.ilargi_norm_grad(None, DY, C, first="none", second="rms", d_h=None, d_x=None, d_gain2=new())[5]
    assert float(want.abs().max()) <= 128 and near(got, want)
    got = il.ilargi_norm_grad(None, DY, C, first="none", second="rms", gate=torch.ones_like(R), d_h=None, d_x=None, d_gate=new(), d_gain1=new(), d_bias1=new(), d_gain2=new(), d_bias2=new())
    assert near(got[5], want) and equal(got[6], dy.to(D).sum(0))


# sizes of the groups (skewed; more than 64; more than 512), inputs, outputs
GROUPED = [([5003], 333, 129), ([20_011, 3, 0, 999], 64, 512), ([2000, 1900, 17, 60], 40, 1031), ([9000, 0, 1, 130] + [3] * 70, 24, 96), ([2] * 300 + [4001] + [1] * 400, 48, 40),
           ([2500, 2100], 1024, 768), ([70_001, 530], 9, 300), ([6000, 700, 7], 512, 2048), ([300, 290, 310, 301, 3, 299, 420, 280], 2048, 2048)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", range(len(GROUPED)))
@pytest.mark.parametrize("act", ["none", "relu"])
def test_sums_of_the_layers_over_rows(il, dtype, case, act):
    sizes, k, m = GROUPED[case]
    n = sum(sizes)
    gen = base._gen(case)
    X, D, pre = _whole((n, k), gen), _whole((n, m), gen), _whole((n, m), gen)
    W = torch.ones(len(sizes), k, m, device="cuda")
    at = [0]
    for s in sizes:
        x, d, z = (t[at[-1]: at[-1] + s] for t in (X, D, pre))
        _halves(x, d, gen, 2)
        z[s - s // 2:] = z[: s // 2]
        at.append(at[-1] + s)
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    dX, dW, db = il.ilargi_grouped_linear_grad(D.to(dtype), X.to(dtype), W.to(dtype), offsets, pre=pre.to(dtype) if act != "none" else None, act=act)
    g = D.double() * (pre > 0) if act == "relu" else D.double()
    if act == "none":
        _seen(g)
    more_W, more_b = torch.ones_like(dW), torch.ones_like(db)
    il.ilargi_grouped_linear_grad(D.to(dtype), X.to(dtype), W.to(dtype), offsets, pre=pre.to(dtype) if act != "none" else None, act=act, d_X=None, d_W=more_W, d_bias=more_b, accumulate=True)
    only_W = il.ilargi_grouped_linear_grad(D.to(dtype), X.to(dtype), W.to(dtype), offsets, pre=pre.to(dtype) if act != "none" else None, act=act, d_X=None, d_bias=None)[1]
    for q in range(len(sizes)):
        rows = slice(at[q], at[q + 1])
        want_W, want_b = X[rows].double().t() @ g[rows], g[rows].sum(0)
        assert float(want_W.abs().max()) < 255 and float(want_b.abs().max()) < 255
        assert torch.equal(dW[q].double(), want_W) and torch.equal(db[q].double(), want_b), q
        assert torch.equal(more_W[q].double(), want_W + 1) and torch.equal(more_b[q].double(), want_b + 1), q
        assert torch.equal(only_W[q].double(), want_W), q
    # (rows of W are ones: what is equal for all k)
    want = g.sum(1, keepdim=True).to(dtype).expand(n, k)
    assert torch.equal(dX, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sums_over_half_a_million_rows(il, dtype):
    """Chunks and parts of a group of 539,300 rows."""
    gen = base._gen(3)
    n, k, m, last = 540_000, 1024, 24, 700
    X, D = _whole((n, k), gen), _whole((n, m), gen)
    _halves(X[: n - last], D[: n - last], gen, 2)
    _halves(X[n - last:], D[n - last:], gen, 2)
    offsets = torch.tensor([0, n - last, n], dtype=torch.int32, device="cuda")
    _, dW, db = il.ilargi_grouped_linear_grad(D.to(dtype), X.to(dtype), torch.ones(2, k, m, dtype=dtype, device="cuda"), offsets, d_X=None)
    for q, rows in enumerate((slice(0, n - last), slice(n - last, n))):
        assert torch.equal(dW[q].double(), X[rows].double().t() @ D[rows].double()) and torch.equal(db[q].double(), D[rows].double().sum(0))
