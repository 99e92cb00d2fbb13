"""Instances of the kernels that only large calls reach: whole blocks of 256 in all three products of a layer, outputs past the caches
of every kind, long runs of sorted keys and segments that reach through many of them."""
import math

import pytest

import test_gpu_linear as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def il():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_01985_amd as mod
    return mod


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# 16 x 16 blocks of 256 and 64 steps of k, the last of them in part, in each of the three products; operands as they lie, and laid out first
@pytest.mark.parametrize("n,k,m,pad,shift", [(4091, 4072, 4088, 0, 0), (4091, 4072, 4088, 8, 8), (4091, 4071, 4087, 3, 1)])
def test_blocks_of_256_over_many_steps(il, n, k, m, pad, shift):
    base.test_forward(il, n, k, m, BF16, pad, shift)
    base.test_gradient(il, n, k, m, BF16, pad, shift)


@pytest.mark.parametrize("n,m,act,keep", [(8209, 8193, "silu", False), (4099, 8200, "none", True)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_outputs_larger_than_the_caches_with_a_residual(il, n, m, act, keep, pad, shift, in_place):
    """Bounds as in the tests of smaller layers; what lies between the rows stays as it was."""
    k, gen = 72, _gen(n + m + pad)
    X, W = base._matrix(n, k, BF16, gen), base._matrix(k, m, BF16, gen, 0, 0, 1 / math.sqrt(k))
    bias, R = torch.randn(m, generator=gen, device="cuda").to(BF16), torch.randn(n, m, generator=gen, device="cuda").to(BF16)
    stores = [torch.full((n * (m + pad) + shift + 8,), 7.0, dtype=BF16, device="cuda") for _ in range(2)]
    out, pre = (s[shift: shift + n * (m + pad)].view(n, m + pad) for s in stores)
    if in_place:
        out[:, :m] = R
    il.ilargi_linear(X, W, bias=bias, residual=out[:, :m] if in_place else R, act=act, out=out[:, :m], pre=pre[:, :m] if keep else None)
    for a in range(0, n, 1024):
        x, r = X[a: a + 1024].double(), R[a: a + 1024].double()
        z = x @ W.double() + bias.double()
        ez = (k + 3) * base.E32 * (x.abs() @ W.double().abs() + bias.double().abs())
        want = base._f(z, act) + r
        err = 1.13 * ez + 16 * base.E32 * (1 + z.abs()) + 2 * base.E32 * (want.abs() + r.abs())
        assert bool(((out[a: a + 1024, :m].double() - want).abs() <= err + base.U[BF16] * (want.abs() + err)).all())
        if keep:
            assert bool(((pre[a: a + 1024, :m].double() - z).abs() <= ez + base.U[BF16] * (z.abs() + ez)).all())
    for s, v in zip(stores, (out, pre)):
        assert bool((v[:, m:] == 7.0).all()) and bool((s[:shift] == 7.0).all()) and bool((s[shift + v.numel():] == 7.0).all())


@pytest.mark.parametrize("dt,do", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("cols,pad,shift", [(256, 0, 0), (264, 8, 8), (250, 0, 0), (257, 3, 1)])
def test_lookups_larger_than_the_caches(il, dt, do, cols, pad, shift):
    """Outputs of 128 MiB and more, whose rows are whole pieces or not: one factor of 0.5 and one rounding, to the bit."""
    n, rows, gen = 300_000, 7000, _gen(cols)
    table = torch.randn(rows, cols, generator=gen, device="cuda").to(dt)
    ids = torch.randint(-1, rows + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
    store = torch.full((n * (cols + pad) + shift + 8,), 7.0, dtype=do, device="cuda")
    out = store[shift: shift + n * (cols + pad)].view(n, cols + pad)
    assert n * cols * out.element_size() >= 128 << 20
    il.ilargi_embed(table, ids, 0.5, out=out[:, :cols])
    live = (ids >= 0) & (ids < rows)
    want = torch.where(live[:, None], table.float()[ids.clamp(0, rows - 1).long()] * 0.5, 0.0).to(do)
    assert torch.equal(out[:, :cols], want)
    assert bool((out[:, cols:] == 7.0).all()) and bool((store[:shift] == 7.0).all()) and bool((store[shift + out.numel():] == 7.0).all())


# keys in runs of 32, 64, 128 and 256; a row that holds them all, or most, reaches through thousands of runs of more than 256 columns
@pytest.mark.parametrize("n,rows,cols,dt,do", [(1_000_000, 100_000, 128, BF16, BF16), (200_001, 3000, 704, F32, F32), (300_007, 500, 1024, BF16, F32),
                                               (600_000, 900, 1100, BF16, BF16), (5003, 40, 300, F32, BF16), (70_001, 6, 515, F32, F32)])
@pytest.mark.parametrize("kind", ["skew", "one", "holes"])
def test_gradients_in_long_runs(il, n, rows, cols, dt, do, kind):
    """Whole numbers, whose sums are exact: the result is their sum, rounded once."""
    gen = _gen(n + cols)
    ids = (torch.rand(n, generator=gen, device="cuda") ** 6 * rows).int().clamp(max=rows - 1)
    if kind == "one":
        ids.fill_(rows // 2)
    if kind == "holes":
        ids[torch.rand(n, generator=gen, device="cuda") < 0.3] = -1
        ids[::7] = rows
    d = torch.randint(-8, 9, (n, cols), generator=gen, device="cuda", dtype=torch.int8).to(dt)
    live = (ids >= 0) & (ids < rows)
    want = torch.zeros(rows, cols, device="cuda")
    for a in range(0, n, 1 << 17):
        part = slice(a, a + (1 << 17))
        want.index_add_(0, ids[part][live[part]].long(), d[part][live[part]].float())
    got = il.ilargi_embed_grad(d, ids, rows, dtype=do)
    assert torch.equal(got, want.to(do))
    old = torch.randint(-8, 9, (rows, cols), generator=gen, device="cuda", dtype=torch.int8).to(do)
    added = il.ilargi_embed_grad(d, ids, rows, scale=-1.0, d_table=old.clone(), accumulate=True)
    assert torch.equal(added, (old.float() - want).to(do))


@pytest.mark.parametrize("k,m", [(8, 8), (64, 256), (264, 136)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_gradient_of_no_rows(il, k, m, dtype):
    """Sums over nothing: zeros, or what was there."""
    X, D = torch.empty(0, k, dtype=dtype, device="cuda"), torch.empty(0, m, dtype=dtype, device="cuda")
    W = torch.randn(k, m, device="cuda").to(dtype)
    d_X, d_W, d_b = il.ilargi_linear_grad(D, X, W, pre=D, act="gelu", d_W=torch.full_like(W, 3.0), d_bias=torch.full((m,), 3.0, dtype=dtype, device="cuda"))
    assert d_X.shape == (0, k) and bool((d_W == 0).all()) and bool((d_b == 0).all())
    old_W, old_b = W.clone(), W[0].clone()
    il.ilargi_linear_grad(D, X, W, d_X=None, d_W=old_W, d_bias=old_b, accumulate=True)
    assert torch.equal(old_W, W) and torch.equal(old_b, W[0])
