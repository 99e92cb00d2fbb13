"""Embedding rows and their gradient against 64 bits.

Unit roundoffs: u32 = 2^-24 for float32, u16 = 2^-8 for bfloat16 (8 significant bits).  A looked-up entry is one product in
float32 (and one sum when accumulating), rounded to the output's type: |err| <= u_out |want| + 2 u32 (|scale x| + |old|) (1 + u_out).
A gradient entry sums c terms in float32 in some order, |err| <= (c + 3) u32 |scale| sum|d| before the one rounding to its type.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def il():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_01985_amd as mod
    return mod


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _matrix(rows, cols, dtype, gen, pad=0, shift=0):
    """A matrix with `pad` columns of NaN beside it, beginning `shift` elements into its storage."""
    store = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    m = store[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
    return m


def _ids(n, rows, kind, gen):
    if rows == 0:
        return torch.full((n,), -1, dtype=torch.int32, device="cuda")
    if kind == "one":
        return torch.full((n,), rows - 1, dtype=torch.int32, device="cuda")
    if kind == "skew":
        ids = (torch.rand(n, generator=gen, device="cuda") ** 6 * rows).int().clamp(max=rows - 1)
    else:
        ids = torch.randint(0, rows, (n,), generator=gen, device="cuda", dtype=torch.int32)
    if kind == "holes":
        ids[torch.rand(n, generator=gen, device="cuda") < 0.3] = -1
        ids[::7] = rows                       # outside the table: takes nothing
        ids[3::11] = -2147483648
        ids[5::13] = 2147483647
    return ids


def _live(ids, rows):
    return (ids >= 0) & (ids < rows)


SHAPES = [(0, 5, 8), (1, 1, 1), (1, 7, 3), (5, 3, 64), (300, 40, 17), (1003, 333, 75), (513, 6040, 128), (64, 2, 1030), (4097, 100, 33)]


@pytest.mark.parametrize("n,rows,cols", SHAPES)
@pytest.mark.parametrize("dt,do", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("kind,pad,shift", [("uniform", 0, 0), ("holes", 3, 1), ("skew", 8, 0)])
def test_lookup(il, n, rows, cols, dt, do, kind, pad, shift):
    gen = _gen(n + 7 * rows + cols)
    table, ids = _matrix(rows, cols, dt, gen, pad, shift), _ids(n, rows, kind, gen)
    out = _matrix(n, cols, do, gen, pad, shift)
    old = out.double()
    beside = torch.as_strided(out, (n, pad), (cols + pad, 1), out.storage_offset() + cols).clone() if pad and n else None
    scale = 1.7
    x = torch.where(_live(ids, rows)[:, None], table.double()[ids.clamp(0, rows - 1).long()] * scale, 0.0)
    for accumulate in (False, True):
        out.copy_(old)
        assert il.ilargi_embed(table, ids, scale, out=out, accumulate=accumulate) is out
        want = x + (old if accumulate else 0.0)
        assert bool(((out.double() - want).abs() <= U[do] * want.abs() + 2.1 * U[F32] * (x.abs() + old.abs())).all())
        if accumulate:
            assert torch.equal(out[~_live(ids, rows)], old[~_live(ids, rows)].to(do))
    if beside is not None:
        after = torch.as_strided(out, (n, pad), (cols + pad, 1), out.storage_offset() + cols)
        assert bool((torch.isnan(after) == torch.isnan(beside)).all())


@pytest.mark.parametrize("n,rows,cols", SHAPES + [(20000, 3, 40), (9001, 200_003, 12), (70_000, 1500, 68)])
@pytest.mark.parametrize("dt,do", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("kind,pad,shift", [("uniform", 0, 0), ("holes", 3, 1), ("skew", 8, 0), ("one", 0, 0)])
def test_gradient(il, n, rows, cols, dt, do, kind, pad, shift):
    gen = _gen(n + 7 * rows + cols)
    d_out, ids = _matrix(n, cols, dt, gen, pad, shift), _ids(n, rows, kind, gen)
    d_table = _matrix(rows, cols, do, gen, pad, shift)
    old = d_table.double()
    scale = 0.9
    live = _live(ids, rows)
    at = ids[live].long()
    d = d_out.double()[live]
    zeros = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    s, t = zeros.index_add(0, at, d) * scale, zeros.index_add(0, at, d.abs()) * scale
    count = torch.bincount(at, minlength=rows)[:, None].double()
    for accumulate in (False, True):
        d_table.copy_(old)
        il.ilargi_embed_grad(d_out, ids, rows, scale, d_table=d_table, accumulate=accumulate)
        want = s + (old if accumulate else 0.0)
        bound = U[do] * want.abs() + 1.01 * U[F32] * ((count + 3) * t + (2 * old.abs() if accumulate else 0.0))
        assert bool(((d_table.double() - want).abs() <= bound).all())
        if accumulate:
            none = count[:, 0] == 0
            assert torch.equal(d_table[none], old[none].to(do))
    again = torch.empty_like(d_table)
    again.copy_(old)
    il.ilargi_embed_grad(d_out, ids, rows, scale, d_table=again, accumulate=True)
    assert torch.equal(again, d_table)                     # the same bits


def test_gradient_is_the_transpose_of_the_lookup(il):
    """<lookup(E), Y> = <E, gradient(Y)>, and differences of the scalar <lookup(E), Y> along a direction (the lookup is linear)."""
    gen = _gen(3)
    n, rows, cols, scale = 2500, 700, 36, 1.25
    E, D = torch.randn(rows, cols, generator=gen, device="cuda"), torch.randn(rows, cols, generator=gen, device="cuda")
    ids, Y = _ids(n, rows, "holes", gen), torch.randn(n, cols, generator=gen, device="cuda")
    G = il.ilargi_embed_grad(Y, ids, rows, scale)
    f = lambda T: float((il.ilargi_embed(T, ids, scale).double() * Y.double()).sum())
    size = float((il.ilargi_embed(D, ids, scale).double() * Y.double()).abs().sum())
    assert abs(f(E) - float((E.double() * G.double()).sum())) <= 1e-5 * float((il.ilargi_embed(E, ids, scale).double() * Y.double()).abs().sum())
    assert abs((f(E + D) - f(E - D)) / 2 - float((D.double() * G.double()).sum())) <= 1e-5 * size


def test_values_that_are_not_finite(il):
    """Infinities and NaN reach the rows that hold them and no others; rows that no key names are zero."""
    gen = _gen(5)
    table = torch.randn(40, 20, generator=gen, device="cuda")
    table[3], table[4], table[5, 7] = float("nan"), float("inf"), -float("inf")
    ids = torch.tensor([3, 0, 4, -1, 5, 40, 1], dtype=torch.int32, device="cuda")
    out = il.ilargi_embed(table, ids, 2.0)
    assert bool(torch.isnan(out[0]).all()) and bool((out[2] == float("inf")).all()) and float(out[4, 7]) == -float("inf")
    assert bool((out[[3, 5]] == 0).all()) and torch.equal(out[[1, 6]], table[[0, 1]] * 2)
    d = torch.ones(7, 20, device="cuda")
    d[3], d[5] = float("nan"), float("inf")              # rows of ids that name nothing
    d[2, 1] = float("nan")
    g = il.ilargi_embed_grad(d, ids, 40)
    assert bool(torch.isnan(g[4, 1])) and int(torch.isnan(g).sum()) == 1 and bool(torch.isfinite(g).sum() == 799)


def test_on_another_stream(il):
    gen = _gen(6)
    ids, d = _ids(5000, 300, "skew", gen), torch.randn(5000, 48, generator=gen, device="cuda")
    want = il.ilargi_embed_grad(d, ids, 300)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = il.ilargi_embed_grad(d, ids, 300, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_in_a_graph(il):
    """Captured once, replayed on new inputs."""
    gen = _gen(8)
    n, rows, cols = 6000, 900, 40
    ids, d = _ids(n, rows, "skew", gen), torch.randn(n, cols, generator=gen, device="cuda")
    out = torch.empty(rows, cols, device="cuda")
    ws = torch.empty(il.ilargi_embed_grad_workspace_bytes(n, rows, cols), dtype=torch.uint8, device="cuda")
    il.ilargi_embed_grad(d, ids, rows, d_table=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        il.ilargi_embed_grad(d, ids, rows, d_table=out, workspace=ws)
    for k in range(4):
        ids.copy_(_ids(n, rows, ("skew", "holes", "one", "uniform")[k], gen))
        d.copy_(torch.randn(n, cols, generator=gen, device="cuda"))
        want = il.ilargi_embed_grad(d, ids, rows)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_workspace_is_enough_and_no_more_is_touched(il):
    gen = _gen(10)
    for n, rows, cols in ((1, 1, 1), (700, 33, 20), (16384, 500, 24), (16385, 500, 24), (60_000, 70_000, 9), (200_000, 3, 40)):
        ids, d = _ids(n, rows, "holes", gen), torch.randn(n, cols, generator=gen, device="cuda")
        nbytes = il.ilargi_embed_grad_workspace_bytes(n, rows, cols)
        store = torch.full((nbytes + 512,), 171, dtype=torch.uint8, device="cuda")
        got = il.ilargi_embed_grad(d, ids, rows, workspace=store[256: 256 + nbytes])
        assert torch.equal(got, il.ilargi_embed_grad(d, ids, rows))
        assert bool((store[:256] == 171).all()) and bool((store[256 + nbytes:] == 171).all())


# every range of the sorts and sums: one workgroup's sort and its border, one to four digits, a row that holds nearly all ids
@pytest.mark.parametrize("n", [1, 63, 64, 65, 1023, 1025, 4096, 16383, 16384, 16385, 40_961])
@pytest.mark.parametrize("rows", [1, 2, 255, 256, 511, 512, 70_000, 300_001])
def test_counts(il, n, rows):
    """Sums of ones are counts: exact."""
    gen = _gen(n + rows)
    for kind in ("uniform", "skew", "one", "holes"):
        ids = _ids(n, rows, kind, gen)
        got = il.ilargi_embed_grad(torch.ones(n, 5, device="cuda"), ids, rows)
        want = torch.bincount(ids[_live(ids, rows)].long(), minlength=rows).float()
        assert torch.equal(got, want[:, None].expand(rows, 5))


def test_refusals(il):
    t = torch.zeros(10, 8, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        il.ilargi_embed(t.half(), ids)
    with pytest.raises(TypeError):
        il.ilargi_embed(t, ids.long())
    with pytest.raises(TypeError):
        il.ilargi_embed(t.t(), ids)
    with pytest.raises(ValueError):
        il.ilargi_embed(t, ids, out=torch.zeros(4, 9, device="cuda"))
    with pytest.raises(ValueError):
        il.ilargi_embed(t, ids, accumulate=True)
    with pytest.raises(ValueError):
        il.ilargi_embed_grad(torch.zeros(5, 8, device="cuda"), ids, 10)
    with pytest.raises(TypeError):
        il.ilargi_embed_grad(torch.zeros(4, 1, device="cuda").expand(4, 8)[:, ::2], ids, 10)
    with pytest.raises(il.IlargiError) as e:
        il.ilargi_embed_grad(torch.zeros(4, 8, device="cuda"), ids, 10, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == il.ERR_WORKSPACE
