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
