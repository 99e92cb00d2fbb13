"""Orthogonalised updates against 64 bits.

A rounding of size e (relative, in the Frobenius norm) in one step is multiplied by at most a = 3.4445 (the slope of
a s + b s^3 + c s^5 at 0, its largest on [0, 1.3]) in every later step.  A step forms three products in float32, each good to
(sqrt(l) + 4) u32 of its size for entries of either sign: e = 3 (sqrt(l) + 4) u32.  So after T steps the result is off by at most
e (a^T - 1) / (a - 1) of the norm that unamplified directions have, which is below that of the result.  bfloat16 results add u16.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16
COEF = (3.4445, -4.7750, 2.0315)


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


def _tol(rows, cols, steps, out):
    a = COEF[0]
    return 3 * (math.sqrt(max(rows, cols)) + 4) * 2.0 ** -24 * (a ** steps - 1) / (a - 1) + (2.0 ** -8 if out == BF16 else 0.0)


def _far(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 1, 9), (1, 9, 1), (3, 5, 7), (2, 16, 16), (4, 220, 64), (1, 64, 220), (2, 33, 65), (1, 129, 127),
                                   (2, 128, 256), (1, 257, 300), (1, 300, 1000), (1, 777, 130), (5, 40, 8), (1, 512, 512)])
@pytest.mark.parametrize("dg,do", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_against_64_bits(il, shape, dg, do, pad):
    b, r, c = shape
    gen = _gen(r + 3 * c + pad)
    wide = torch.full((b, r, c + pad), float("nan"), device="cuda").to(dg)
    G = wide[:, :, :c]
    rank = max(1, min(r, c) // 4)
    low = torch.randn(b, r, rank, generator=gen, device="cuda") @ torch.randn(b, rank, c, generator=gen, device="cuda")
    G.copy_((low + torch.randn(b, r, c, generator=gen, device="cuda")) * 1e-3)
    out = torch.full((b, r, c + pad), float("nan"), device="cuda").to(do)[:, :, :c]
    for steps in (1, 5):
        want = _exact(G, steps)
        assert il.ilargi_orthogonalize(G, out=out, steps=steps) is out
        for q in range(b):
            assert _far(out[q], want[q]) <= _tol(r, c, steps, do)
    again = il.ilargi_orthogonalize(G, steps=5, out_dtype=do)
    assert torch.equal(again, out)
    assert bool(torch.isnan(wide[:, :, c:]).all())


def test_singular_values_come_near_one(il):
    gen = _gen(1)
    for r, c in ((96, 96), (200, 64)):
        s = torch.linalg.svdvals(il.ilargi_orthogonalize(torch.randn(r, c, generator=gen, device="cuda")).double())
        assert float(s.max()) < 1.3 and float((s > 0.6).double().mean()) > 0.9


def test_updates_weights_in_place(il):
    gen = _gen(2)
    for dtype in (F32, BF16):
        for r, c in ((70, 41), (64, 128)):
            W = torch.randn(r, c, generator=gen, device="cuda").to(dtype)
            G = torch.randn(r, c, generator=gen, device="cuda") * 1e-2
            want = 0.99 * W.double() - 0.3 * _exact(G, 5)
            got = il.ilargi_orthogonalize(G, out=W, base=W, alpha=-0.3, beta=0.99)
            assert got is W and _far(W, want) <= _tol(r, c, 5, dtype)


def test_coefficients_and_scale(il):
    """Cubic Newton-Schulz (3/2, -1/2, 0) converges to the orthogonal factor; the result does not depend on the scale of G."""
    gen = _gen(3)
    G = torch.randn(48, 80, generator=gen, device="cuda")
    U, _, Vh = torch.linalg.svd(G.double(), full_matrices=False)
    out = il.ilargi_orthogonalize(G, steps=40, coef=(1.5, -0.5, 0.0))
    # at the fixed point an error along the factor is halved away and one across it stays: forty steps add at most forty roundings
    assert _far(out, U @ Vh) <= 40 * 3 * (math.sqrt(80) + 4) * 2.0 ** -24
    for scale in (1e-30, 1e-10, 1e10, 1e30, 3e37):
        x = G * scale / 8
        assert _far(il.ilargi_orthogonalize(x, eps=0.0), _exact(x, 5, eps=0.0)) <= _tol(48, 80, 5, F32)


def test_coefficients_that_leave_the_unit_interval(il):
    """a = 4, b = c = 0 multiplies by 4 a step (A^2 stays below 2e19); 3 s - 30 s^3 leaves every interval."""
    G = torch.randn(70, 40, generator=_gen(7), device="cuda")
    for steps, coef in ((8, (4.0, 0.0, 0.0)), (3, (3.0, -30.0, 1.0))):
        assert _far(il.ilargi_orthogonalize(G, steps=steps, coef=coef), _exact(G, steps, coef)) <= 1e-4


def test_zero_and_values_that_are_not_finite(il):
    G = torch.zeros(3, 20, 33, device="cuda")
    G[1] = torch.randn(20, 33, generator=_gen(4), device="cuda")
    G[2] = G[1]
    G[2, 4, 5] = float("nan")
    out = il.ilargi_orthogonalize(G)
    assert bool((out[0] == 0).all()) and bool(torch.isnan(out[2]).any())
    assert _far(out[1], _exact(G[1], 5)) <= _tol(20, 33, 5, F32)          # its neighbours leave it alone
    G[2, 4, 5] = float("inf")
    assert not bool(torch.isfinite(il.ilargi_orthogonalize(G)[2]).all())
    base = torch.full((3, 20, 33), float("nan"), device="cuda")
    assert bool(torch.isfinite(il.ilargi_orthogonalize(G[:2], out=base[:2], base=base[:2], beta=0.0)).all())   # beta 0: not read


def test_on_another_stream_and_in_a_graph(il):
    gen = _gen(5)
    for dtype, shape in ((F32, (2, 72, 40)), (BF16, (1, 136, 264))):
        G = torch.randn(shape, generator=gen, device="cuda").to(dtype)
        out = torch.empty_like(G)
        ws = torch.empty(il.ilargi_orthogonalize_workspace_bytes(*shape, dtype), dtype=torch.uint8, device="cuda")
        want = il.ilargi_orthogonalize(G)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        il.ilargi_orthogonalize(G, out=out, workspace=ws, stream=side)
        side.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            il.ilargi_orthogonalize(G, out=out, workspace=ws)
        for _ in range(3):
            G.copy_(torch.randn(shape, generator=gen, device="cuda"))
            want = il.ilargi_orthogonalize(G)
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_workspace_is_enough_and_no_more_is_touched(il):
    gen = _gen(9)
    for shape in ((2, 40, 300), (3, 65, 65), (1, 500, 1100), (1, 1030, 520), (5, 130, 130)):
        for dtype in (F32, BF16):
            G = torch.randn(shape, generator=gen, device="cuda").to(dtype)
            nbytes = il.ilargi_orthogonalize_workspace_bytes(*shape, dtype)
            store = torch.full((nbytes + 512,), 171, dtype=torch.uint8, device="cuda")
            for coef in (None, (2.0, -3.0, 9.0)):           # in pairs, and where the iteration leaves them
                steps = 5 if coef is None else 2
                got = il.ilargi_orthogonalize(G, steps=steps, coef=coef, workspace=store[256: 256 + nbytes])
                assert _far(got, _exact(G, steps, coef or COEF)) <= 1e-2
                assert bool((store[:256] == 171).all()) and bool((store[256 + nbytes:] == 171).all())


def test_refusals(il):
    G = torch.zeros(8, 6, device="cuda")
    with pytest.raises(TypeError):
        il.ilargi_orthogonalize(G.double())
    with pytest.raises(ValueError):
        il.ilargi_orthogonalize(G[0])
    with pytest.raises(TypeError):
        il.ilargi_orthogonalize(G.t())
    with pytest.raises(ValueError):
        il.ilargi_orthogonalize(G, out=torch.zeros(6, 8, device="cuda"))
    with pytest.raises(ValueError):
        il.ilargi_orthogonalize(G, beta=0.5)
    for steps in (0, -1, 101):
        with pytest.raises(il.IlargiError) as e:
            il.ilargi_orthogonalize(G, steps=steps)
        assert e.value.status == il.ERR_SHAPE
    with pytest.raises(il.IlargiError) as e:
        il.ilargi_orthogonalize(G, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == il.ERR_WORKSPACE
