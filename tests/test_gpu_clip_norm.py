"""The norm over many tensors, and the tensors scaled by it, against 64 bits.

Squares and their sums are float64: the norm is off by its rounding to float32, E = 2^-24 of itself (and 2^-50).  A scaled value is x times a
factor of 24 bits (E), rounded in float32 (E) and to its type (u): (2 E + u) of itself, plus the least float32 number where it is subnormal.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
E = 2.0 ** -24


@pytest.fixture(scope="module")
def il():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_01985_amd as mod
    return mod


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _norm64(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


def _check(il, tensors, max_norm, outs, norm, old):
    want = _norm64(old)
    assert abs(float(norm) - want) <= 1.01 * E * want
    factor = min(1.0, max_norm / want) if want > 0 else 1.0
    for t, o, was in zip(tensors, outs, old):
        if factor == 1.0:
            assert torch.equal(o, was)
        else:
            exact = was.double() * factor
            assert bool(((o.double() - exact).abs() <= 1.01 * (2 * E + U[o.dtype]) * exact.abs() + 1.5e-45 + (9.2e-41 if o.dtype == BF16 else 0.0)).all())


SHAPES = [[(1,)], [(7,), (3, 5)], [(64, 64), (64,), (64, 256), (22, 7)], [(1000, 33), (0,), (5, 0), (129,), (2, 3, 5)], [(300_001,), (1,), (17, 4096)], [(9,)] * 200, [(2048, 2048), (2048,)] * 3]


@pytest.mark.parametrize("case", range(len(SHAPES)))
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
def test_norm_and_scaling(il, case, kind):
    gen = _gen(case)
    types = {"f32": [F32], "bf16": [BF16], "mixed": [BF16, F32, F32]}[kind]
    tensors = [torch.randn(s, generator=gen, device="cuda").to(types[q % len(types)]) for q, s in enumerate(SHAPES[case])]
    old, norm64 = [t.clone() for t in tensors], _norm64(tensors)
    for max_norm in (0.37 * norm64, 2.0 * norm64, math.inf, 0.0):
        max_norm = float(torch.tensor(max_norm))
        outs = [torch.full_like(t, 5.0) for t in tensors]
        norm = il.ilargi_clip_norm(il.TensorList(tensors, outs), max_norm)
        _check(il, tensors, max_norm, outs, norm, old)
        assert all(torch.equal(t, o) for t, o in zip(tensors, old))
        again = il.ilargi_clip_norm(il.TensorList(tensors), max_norm)                       # the norm alone
        assert torch.equal(again, norm) and all(torch.equal(t, o) for t, o in zip(tensors, old))
        inplace = [t.clone() for t in tensors]
        assert torch.equal(il.ilargi_clip_norm(inplace, max_norm), norm)
        assert all(torch.equal(a, b) for a, b in zip(inplace, outs))
    # some of them are not written
    max_norm = float(torch.tensor(0.5 * norm64))
    some = [torch.empty_like(t) if q % 2 == 0 else None for q, t in enumerate(tensors)]
    norm = il.ilargi_clip_norm(il.TensorList(tensors, some), max_norm)
    every = [torch.empty_like(t) for t in tensors]
    assert torch.equal(il.ilargi_clip_norm(il.TensorList(tensors, every), max_norm), norm)
    assert all(o is None or torch.equal(o, e) for o, e in zip(some, every)) and all(torch.equal(t, o) for t, o in zip(tensors, old))


def test_no_tensors(il):
    assert float(il.ilargi_clip_norm([], 1.0)) == 0.0
    assert float(il.ilargi_clip_norm([torch.empty(0, device="cuda")], 1.0)) == 0.0
    zeros = [torch.zeros(5, 3, device="cuda")]
    assert float(il.ilargi_clip_norm(zeros, 0.0)) == 0.0 and bool((zeros[0] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_addresses(il, dtype):
    """Column slices of one matrix beside each other, rows of a batch, a strided vector, addresses of single elements; what lies between
    is left alone."""
    gen = _gen(6)
    wide = torch.randn(40, 100, generator=gen, device="cuda").to(dtype)
    cube = torch.randn(3, 5, 20, generator=gen, device="cuda").to(dtype)
    long = torch.randn(1001, generator=gen, device="cuda").to(dtype)
    views = lambda w, c, v: [w[:, :33], w[:, 33:60], w[:20, 61:99], w[5, 99:], c[:, :, 3:18], v[1:400], v[401::3]]
    tensors = views(wide, cube, long)
    old, norm64 = [t.clone() for t in tensors], _norm64(tensors)
    max_norm = float(torch.tensor(0.3 * norm64))
    outs = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in tensors]
    norm = il.ilargi_clip_norm(il.TensorList(tensors, outs), max_norm)
    _check(il, tensors, max_norm, outs, norm, old)
    stores = [wide.clone(), cube.clone(), long.clone()]
    assert torch.equal(il.ilargi_clip_norm(views(*stores), max_norm), norm)
    for got, was, views_of in zip(stores, (wide, cube, long), range(3)):
        touched = torch.zeros_like(got, dtype=torch.bool)
        marks = [torch.zeros_like(t, dtype=torch.bool) for t in (wide, cube, long)]
        for t in views(*marks):
            t.fill_(True)
        touched = marks[views_of]
        assert torch.equal(got[~touched], was[~touched])
    assert all(torch.equal(a, b) for a, b in zip(views(*stores), outs))
    # strided outputs of contiguous tensors
    back = [torch.randn(40, 100, generator=gen, device="cuda").to(dtype), torch.randn(3, 5, 20, generator=gen, device="cuda").to(dtype), torch.randn(1001, generator=gen, device="cuda").to(dtype)]
    flat = [t.contiguous() for t in tensors]
    il.ilargi_clip_norm(il.TensorList(flat, views(*back)), max_norm)
    _check(il, flat, max_norm, views(*back), norm, old)


def test_large_and_small_entries(il):
    """Squares that no float32 holds, sums that leave its range, factors below 2^-126."""
    for dtype in (F32, BF16):
        big, small = torch.full((300,), 1e38, device="cuda").to(dtype), torch.full((70,), 1e-30, device="cuda").to(dtype)
        norm = il.ilargi_clip_norm(il.TensorList([small]), 1.0)
        assert abs(float(norm) - _norm64([small])) <= 1.01 * E * _norm64([small])
        out = [torch.empty_like(big)]
        norm = il.ilargi_clip_norm(il.TensorList([big], out), 1e-3)
        assert math.isinf(float(norm))                                        # sqrt(300) 1e38 is no float32 number
        want = big.double() * (float(torch.tensor(1e-3)) / _norm64([big]))
        assert bool(((out[0].double() - want).abs() <= 1.01 * (2 * E + U[dtype]) * want.abs()).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_norms_that_are_not_finite_scale_nothing(il, bad):
    gen = _gen(9)
    tensors = [torch.randn(s, generator=gen, device="cuda") for s in ((50, 60), (7,))]
    tensors[0][3, 4] = bad
    old, outs = [t.clone() for t in tensors], [torch.zeros_like(t) for t in tensors]
    norm = il.ilargi_clip_norm(il.TensorList(tensors, outs), 0.5)
    assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf
    same = lambda a, b: torch.equal(a.view(torch.int32), b.view(torch.int32))
    assert all(same(o, t) for o, t in zip(outs, old))
    il.ilargi_clip_norm(tensors, 0.5)
    assert all(same(o, t) for o, t in zip(tensors, old))


def test_on_another_stream_and_in_a_graph(il):
    gen = _gen(12)
    tensors = [torch.randn(300, 40, generator=gen, device="cuda").bfloat16(), torch.randn(5000, generator=gen, device="cuda")] + [torch.randn(9, generator=gen, device="cuda") for _ in range(80)]
    outs = [torch.empty_like(t) for t in tensors]
    kept, norm = il.TensorList(tensors, outs), torch.empty(1, device="cuda")
    nbytes = il.ilargi_clip_norm_workspace_bytes(kept)
    store = torch.full((nbytes + 512,), 171, dtype=torch.uint8, device="cuda")
    ws = store[256: 256 + nbytes]
    step = lambda stream=None: il.ilargi_clip_norm(kept, 3.0, norm=norm, workspace=ws, stream=stream)
    step()
    want = [norm.clone(), *(o.clone() for o in outs)]
    side = torch.cuda.Stream()
    for o in outs:
        o.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, [norm, *outs]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for q in range(3):
        tensors[0].copy_(torch.randn(300, 40, generator=gen, device="cuda") * 10.0 ** (q - 2))
        tensors[1].mul_(0.01)
        step()
        want = [norm.clone(), *(o.clone() for o in outs)]
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [norm, *outs]))
    assert bool((store[:256] == 171).all()) and bool((store[256 + nbytes:] == 171).all())


def test_python_refuses(il):
    a = torch.zeros(6, 8, device="cuda")
    for call in (lambda: il.TensorList([a], [a[:5]]), lambda: il.TensorList([a], [a.bfloat16()]), lambda: il.TensorList([a], [])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: il.TensorList([a.half()]), lambda: il.TensorList([a.t()]), lambda: il.TensorList([a[:1].expand(6, 8)]), lambda: il.TensorList([torch.zeros(3)])):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: il.ilargi_clip_norm([a, a], 1.0), lambda: il.ilargi_clip_norm([a, a[2:]], 1.0), lambda: il.ilargi_clip_norm([a], -1.0), lambda: il.ilargi_clip_norm([a], math.nan),
                 lambda: il.ilargi_clip_norm(il.TensorList([a[1:]], [a[:-1]]), 1.0)):
        with pytest.raises(il.IlargiError):
            call()
    assert float(il.ilargi_clip_norm(il.TensorList([a, a]), 1.0)) == 0.0           # counted twice
