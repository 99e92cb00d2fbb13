"""Calls of the operators with learned features whose rows, columns or outputs are so many that one launch cannot have a thread for
each: the header takes up to 2^31 - 1 of either.  Values are chosen so that every result is exact, or repeats from chunk to chunk.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def il():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_01985_amd as mod
    return mod


@pytest.fixture(autouse=True)
def _give_back():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def _room(gib):
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip(f"{gib} GiB of device memory are not free")


def _ints(shape, seed, most=8):
    """Small whole numbers: their products and sums are exact in float32, and they are numbers of bfloat16."""
    return torch.randint(-most, most + 1, shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("accumulate", [False, True])
def test_lookup_of_many_wide_rows(il, accumulate):
    """2^26 + 3 rows of 257 columns: 64 lanes a row are more than 2^32."""
    _room(48)
    n, rows, cols, chunk = (1 << 26) + 3, 37, 257, 1 << 20
    table = _ints((rows, cols), 1).to(BF16)
    ids = (torch.arange(n, device="cuda", dtype=torch.int32) * 7 + torch.arange(n, device="cuda", dtype=torch.int32) // 1000) % (rows + 1)
    ids[ids == rows] = -1
    out = torch.full((n, cols), 2.0, dtype=BF16, device="cuda")
    il.ilargi_embed(table, ids, 1.0, out=out, accumulate=accumulate)
    padded = torch.cat([table, torch.zeros(1, cols, dtype=BF16, device="cuda")])
    for a in range(0, n, chunk):
        want = padded[ids[a: a + chunk].long()] + (2.0 if accumulate else 0.0)
        assert torch.equal(out[a: a + chunk], want)


def test_gradient_of_a_table_of_many_rows(il):
    """2^30 + 5 rows: a workgroup for 256 of them each."""
    _room(8)
    rows, n = (1 << 30) + 5, 5000
    d = _ints((n, 1), 2).to(BF16)
    ids = (_ints((n,), 3, 1 << 20).long().abs() * 1024).clamp(max=rows - 1).int()
    ids[:3], ids[3], ids[4:9] = rows - 1, 0, torch.tensor([rows - 2, rows, -1, 1 << 29, rows - 6], dtype=torch.int32, device="cuda")
    got = il.ilargi_embed_grad(d, ids, rows, d_table=torch.full((rows, 1), 3.0, dtype=BF16, device="cuda"))
    live = (ids >= 0) & (ids < rows)
    want = torch.zeros(rows, dtype=BF16, device="cuda")
    at, inverse = ids[live].long().unique(return_inverse=True)
    want[at] = torch.zeros(at.numel(), device="cuda").index_add_(0, inverse, d[live, 0].float()).to(BF16)
    assert torch.equal(got[:, 0], want)


@pytest.mark.parametrize("accumulate", [False, True])
def test_rows_of_very_many_columns(il, accumulate):
    """2^24 + 100 columns: more slabs of 256 than a launch has along its second axis."""
    _room(4)
    n, rows, cols = 5, 3, (1 << 24) + 100
    d, ids = _ints((n, cols), 4).float(), torch.tensor([2, 0, 2, -1, 0], dtype=torch.int32, device="cuda")
    old = _ints((rows, cols), 5).float()
    got = il.ilargi_embed_grad(d, ids, rows, d_table=old.clone(), accumulate=accumulate)
    want = torch.stack([d[1] + d[4], torch.zeros_like(d[0]), d[0] + d[2]]) + (old if accumulate else 0.0)
    assert torch.equal(got, want)
    assert torch.equal(il.ilargi_embed(got, ids, 1.0)[:3], got[[2, 0, 2]])


@pytest.mark.parametrize("n,k,m,dtype,gib", [
    ((1 << 26) + 9, 257, 1, BF16, 80),        # operands laid out first, 64 lanes a row
    ((1 << 30) + 3, 17, 1, F32, 90),          # blocks of 64 rows
    ((1 << 31) - 1, 8, 8, BF16, 120),          # blocks of 128 rows on the 16-bit matrix cores
])
def test_layers_of_many_rows(il, n, k, m, dtype, gib):
    """The same rows again and again: every chunk of the result is the first one."""
    _room(gib)
    chunk = 1 << 22
    X = torch.empty(n, k, dtype=dtype, device="cuda")
    first, W, bias = _ints((chunk, k), 6, 3).to(dtype), _ints((k, m), 7, 3).to(dtype), _ints((m,), 8, 3).to(dtype)
    for a in range(0, n, chunk):
        X[a: a + chunk] = first[: n - a]
    out = torch.empty(n, m, dtype=dtype, device="cuda")
    il.ilargi_linear(X, W, bias=bias, act="relu", out=out)
    want = (first.float() @ W.float() + bias.float()).clamp(min=0).to(dtype)
    for a in range(0, n, chunk):
        assert torch.equal(out[a: a + chunk], want[: n - a]), a


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_row_of_many_outputs(il, dtype):
    """2^28 + 3 columns of W, two of X; the gradient of the bias and of the inputs."""
    _room(16)
    k, m = 2, (1 << 28) + 3
    X, W, bias = _ints((1, k), 9).to(dtype), _ints((k, m), 10).to(dtype), _ints((m,), 11).to(dtype)
    out = il.ilargi_linear(X, W, bias=bias)
    want = (X[0, 0].float() * W[0].float() + X[0, 1].float() * W[1].float() + bias.float()).to(dtype)
    assert torch.equal(out[0], want)
    d_bias = il.ilargi_linear_grad(W, torch.zeros(k, 1, dtype=dtype, device="cuda"), W[:1], d_X=None, d_W=None)[2]
    assert torch.equal(d_bias, (W[0].float() + W[1].float()).to(dtype))


def test_many_outputs_of_several_rows(il):
    """2^30 + 1 columns for five rows: blocks of 64 side by side."""
    _room(110)
    n, k, m, chunk = 5, 17, (1 << 30) + 1, 1 << 22
    X, first, W = _ints((n, k), 12, 3).float(), _ints((k, chunk), 13, 3).float(), torch.empty(k, m, device="cuda")
    for a in range(0, m, chunk):
        W[:, a: a + chunk] = first[:, : m - a]
    out = il.ilargi_linear(X, W)
    want = X @ first
    for a in range(0, m, chunk):
        assert torch.equal(out[:, a: a + chunk], want[:, : m - a]), a
