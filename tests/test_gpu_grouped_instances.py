"""Layers by group: every kernel that a rule may choose, at sizes that reach it, and calls side by side."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import test_gpu_grouped as base  # noqa: E402
from test_gpu_grouped import BF16, E, F32, U, _f, _gen, _matrices, _matrix, _offsets, _slope, _within, il  # noqa: E402,F401


def _check(il, sizes, k, m, dtype, pad=0, shift=0, act="gelu", residual=False, seed=0):
    G, n = len(sizes), sum(sizes) + 2
    gen = _gen(seed)
    X, W = _matrix(n, k, dtype, gen, pad, shift), _matrices(G, k, m, dtype, gen, pad, shift, k ** -0.5)
    b, R, D, Z, out, pre = _matrix(G, m, dtype, gen, pad, shift), *(_matrix(n, m, dtype, gen, pad, shift) for _ in range(5))
    dX, dW, db = _matrix(n, k, dtype, gen, pad, shift), _matrices(G, k, m, dtype, gen, pad, shift), _matrix(G, m, dtype, gen, pad, shift)
    offsets = _offsets(sizes, 1)
    at = offsets.tolist()
    before = out.clone(), dX.clone()
    il.ilargi_grouped_linear(X, W, offsets, bias=b, residual=R if residual else None, act=act, out=out, pre=pre)
    il.ilargi_grouped_linear_grad(D, X, W, offsets, pre=Z if act != "none" else None, act=act, d_X=dX, d_W=dW, d_bias=db)
    ug = U[dtype] if dtype == BF16 and act != "none" else 0.0
    slack = 0.0 if act == "none" else 32 * E
    for g in range(G):
        s, rows = slice(at[g], at[g + 1]), sizes[g]
        x, w, d = X[s].double(), W[g].double(), D[s].double()
        z = x @ w + b[g].double()
        ez = (k + 3) * E * (x.abs() @ w.abs() + b[g].double().abs())
        f = _f(z, act)
        want = f + (R[s].double() if residual else 0.0)
        _within(out[s], want, 1.13 * ez + (0.0 if act == "none" else 16 * E * (1 + z.abs())) + E * (want.abs() + f.abs()), dtype, ("out", g))
        _within(pre[s], z, ez, dtype, ("pre", g))
        grad = d * _slope(Z[s].double(), act)
        for name, got, want, size, raw, r, rounded in (
                ("d_X", dX[s], grad @ w.t(), grad.abs() @ w.t().abs(), d.abs() @ w.t().abs(), m, ug),
                ("d_W", dW[g], x.t() @ grad, x.t().abs() @ grad.abs(), x.t().abs() @ d.abs(), rows, ug),
                ("d_b", db[g], grad.sum(0), grad.abs().sum(0), d.abs().sum(0), rows, 0.0)):
            _within(got, want, size * (rounded + (r + 4) * E) * 1.01 + 1.01 * slack * raw, dtype, (name, g))
    for new, old in zip((out, dX), before):
        assert torch.equal(new[:1], old[:1]) and torch.equal(new[n - 1:], old[n - 1:])


# rounds of large blocks with a last one that is split over k (304 blocks), one that is not (448), less than one round; forward and back
@pytest.mark.parametrize("sizes,k,m", [([3000, 1400, 100], 1024, 4096), ([3000, 1400, 100], 4096, 1024), ([3000, 2500, 100, 1, 900], 512, 4096), ([1100, 0, 900], 2048, 1032),
                                       ([5000, 300], 1000, 2056)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8)])
def test_rounds_of_large_blocks(il, sizes, k, m, pad, shift):
    _check(il, sizes, k, m, BF16, pad, shift, residual=pad > 0)


# few rows in most groups, many in one of them; lengths of k that end inside a step, columns that end inside a block; shares of k
@pytest.mark.parametrize("sizes,k,m", [([100, 1, 1, 1, 1, 0, 0, 2], 328, 136), ([1], 4096, 64), ([31, 33, 32, 1], 1032, 72), ([3] * 64, 64, 64), ([2] * 65, 200, 72), ([0, 0, 7], 8, 8),
                                       ([20, 1, 24], 2048, 2048), ([200] + [0, 1] * 40, 520, 520)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (1, 3)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_few_rows(il, sizes, k, m, pad, shift, dtype):
    _check(il, sizes, k, m, dtype, pad, shift, act="silu", residual=pad == 8)


# as many groups as there are lanes, one more, and one less; the longest first or as they come
@pytest.mark.parametrize("groups", [1, 2, 63, 64, 65, 130])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_groups_in_lanes(il, groups, dtype):
    sizes = [(7 * g * g + 3) % 71 if g % 5 else 0 for g in range(groups)]
    sizes[groups // 2] = 700
    _check(il, sizes, 72, 88, dtype, act="sigmoid")
    _check(il, sizes, 33, 129, dtype, act="none", pad=1, shift=1)


def test_one_group_is_the_layer(il):
    """The same layer by ilargi_linear: the same sums in other orders."""
    gen = _gen(5)
    for dtype in (F32, BF16):
        n, k, m = 900, 136, 264
        X, W, D = _matrix(n, k, dtype, gen), _matrices(1, k, m, dtype, gen, scale=0.1), _matrix(n, m, dtype, gen)
        o = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        size = X.double().abs() @ W[0].double().abs()
        a, b = il.ilargi_grouped_linear(X, W, o), il.ilargi_linear(X, W[0])
        assert bool(((a.double() - b.double()).abs() <= 2 * (k + 3) * E * size + 2.02 * U[dtype] * b.double().abs()).all())
        for p, q, size, r in zip(il.ilargi_grouped_linear_grad(D, X, W, o), il.ilargi_linear_grad(D, X, W[0]),
                                 (D.double().abs() @ W[0].double().abs().t(), X.double().abs().t() @ D.double().abs(), D.double().abs().sum(0)), (m, n, n)):
            p = p[0] if p.dim() > q.dim() else p
            assert bool(((p.double() - q.double()).abs() <= 2 * (r + 4) * E * size + 2.02 * U[dtype] * q.double().abs()).all())


def test_calls_on_two_streams_at_once(il):
    """Each with a workspace of its own: the same bits as one after the other."""
    gen = _gen(6)
    calls = []
    for dtype, sizes, k, m in ((BF16, [2000, 30, 900], 512, 1024), (F32, [400, 0, 90, 3], 200, 129)):
        n, G = sum(sizes), len(sizes)
        X, W, D, o = _matrix(n, k, dtype, gen), _matrices(G, k, m, dtype, gen, scale=0.1), _matrix(n, m, dtype, gen), _offsets(sizes, 0)
        ws = torch.empty(max(il.ilargi_grouped_linear_workspace_bytes(G, n, k, m, dtype)), dtype=torch.uint8, device="cuda")
        calls.append((X, W, D, o, ws, torch.cuda.Stream(), (torch.empty_like(X), torch.empty_like(W), torch.empty(G, m, dtype=dtype, device="cuda"), torch.empty_like(D))))

    def go(X, W, D, o, ws, stream, res):
        il.ilargi_grouped_linear(X, W, o, out=res[3], act="gelu", workspace=ws, stream=stream)
        il.ilargi_grouped_linear_grad(D, X, W, o, pre=D, act="gelu", d_X=res[0], d_W=res[1], d_bias=res[2], workspace=ws, stream=stream)

    want = []
    for c in calls:
        go(*c)
        torch.cuda.synchronize()
        want.append([t.clone() for t in c[6]])
    for _ in range(3):
        for c in calls:
            for t in c[6]:
                t.zero_()
        torch.cuda.synchronize()
        for c in calls:
            go(*c)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for w, c in zip(want, calls) for a, b in zip(w, c[6]))


def test_matrices_beside_each_other(il):
    """The matrices of the groups as column blocks of one, whose rows interleave, are refused; rows apart are not."""
    n, k, m = 12, 8, 16
    X, o = torch.randn(n, k, device="cuda"), _offsets([5, 7], 0)
    wide = torch.randn(k, 2 * m, device="cuda")
    with pytest.raises(TypeError):
        il.ilargi_grouped_linear(X, wide.view(k, 2, m).transpose(0, 1), o)
    tall = torch.randn(2, k + 3, m + 5, device="cuda")
    W = tall[:, 2:-1, 1: m + 1]
    assert torch.equal(il.ilargi_grouped_linear(X, W, o), il.ilargi_grouped_linear(X, W.contiguous(), o))
