"""Layers by group of rows and their gradients against 64 bits; the bounds are those of one layer (test_gpu_linear.py), group by group.

With E = 2^-24 and u half a step of the layer's type.  z: |err| <= (k + 3) E (sum|x||w| + |bias|).  f: slope at most 1.13, good to
16 E (1 + |z|).  A stored value adds u of itself.  Gradients: g = d f'(z) with f' good to 32 E, rounded to the type (u); sums of r products:
sum|g||w| (u [bf16] + (r + 4) E) + 32 E sum|d||w|; parts of rows that are added add nothing to that, as r + 4 counts every addition.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
E = 2.0 ** -24
ACTS = ["none", "relu", "sigmoid", "silu", "gelu"]


@pytest.fixture(scope="module")
def il():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_01985_amd as mod
    return mod


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _matrix(rows, cols, dtype, gen, pad=0, shift=0, scale=1.0):
    store = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    m = store[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=gen, device="cuda") * scale)
    return m


def _matrices(groups, k, m, dtype, gen, pad=0, shift=0, scale=1.0):
    """groups x k x m, with `pad` rows between the matrices and `pad` columns between their rows."""
    far = (k + pad) * (m + pad)
    store = torch.full((groups * far + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    w = store[shift: shift + groups * far].view(groups, k + pad, m + pad)[:, :k, :m]
    w.copy_(torch.randn(groups, k, m, generator=gen, device="cuda") * scale)
    return w


def _f(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "sigmoid":
        return torch.sigmoid(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "sigmoid":
        return torch.sigmoid(z) * torch.sigmoid(-z)
    if act == "silu":
        return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    if act == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def _within(got, want, err, dtype, name):
    off = (got.double() - want).abs() - (err + U[dtype] * (want.abs() + err)) - 1e-37
    assert bool((off <= 0).all()), (name, float(off.max()) if off.numel() else 0.0)


# sizes of the groups (with rows before the first and behind the last), inputs, outputs
CASES = [
    ([1], 0, 0, 1, 1), ([0], 2, 1, 3, 5), ([3, 0, 1, 7], 0, 0, 5, 3), ([1, 1, 1, 1, 0, 1], 0, 3, 64, 96), ([0, 5, 0, 0, 130, 1], 4, 9, 40, 72), ([2] * 70, 0, 0, 24, 40),
    ([64, 65, 63, 128, 129, 127], 0, 5, 72, 136), ([300, 0, 17], 1, 1, 333, 129), ([256, 257, 1], 0, 0, 264, 520), ([900, 3, 40], 7, 0, 128, 256), ([1] * 8, 0, 0, 1000, 333),
    ([700], 0, 2, 96, 64), ([33, 1500, 8, 0, 90], 3, 3, 200, 104), ([5] * 600, 0, 1, 8, 16), ([8, 8], 0, 0, 2048, 512),
]


def _offsets(sizes, before):
    return torch.tensor([before] + [before + sum(sizes[: q + 1]) for q in range(len(sizes))], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (3, 1)])
def test_forward(il, case, dtype, pad, shift):
    sizes, before, behind, k, m = CASES[case]
    G, n = len(sizes), before + sum(sizes) + behind
    gen = _gen(case + 17 * pad)
    X, W = _matrix(n, k, dtype, gen, pad, shift), _matrices(G, k, m, dtype, gen, pad, shift, 1 / math.sqrt(k))
    bias, R, out, pre = _matrix(G, m, dtype, gen, pad, shift), *(_matrix(n, m, dtype, gen, pad, shift) for _ in range(3))
    offsets = _offsets(sizes, before)
    at = offsets.tolist()
    if before:
        X[:before] = float("nan")
    if behind:
        X[n - behind:] = float("inf")
    for q, act in enumerate(ACTS):
        b, r, keep = (bias if q != 1 else None), (R if q % 2 == 0 else None), q != 3
        old_out, old_pre = out.clone(), pre.clone()
        got = il.ilargi_grouped_linear(X, W, offsets, bias=b, residual=r, act=act, out=out, pre=pre if keep else None)
        assert got is out
        for g in range(G):
            s = slice(at[g], at[g + 1])
            z = X[s].double() @ W[g].double() + (b[g].double() if b is not None else 0.0)
            ez = (k + 3) * E * (X[s].double().abs() @ W[g].double().abs() + (b[g].double().abs() if b is not None else 0.0))
            f = _f(z, act)
            want = f + (r[s].double() if r is not None else 0.0)
            _within(out[s], want, 1.13 * ez + (0.0 if act == "none" else 16 * E * (1 + z.abs())) + E * (want.abs() + f.abs()), dtype, (act, g))
            if keep:
                _within(pre[s], z, ez, dtype, ("pre", act, g))
        for new, old in ((out, old_out), (pre, old_pre)):
            assert torch.equal(new[:before], old[:before]) and torch.equal(new[n - behind:], old[n - behind:])
    first = il.ilargi_grouped_linear(X, W, offsets, bias=bias, residual=R, act="silu")
    assert bool((first[:before] == 0).all()) and bool((first[n - behind:] == 0).all())
    out.copy_(R)
    il.ilargi_grouped_linear(X, W, offsets, bias=bias, residual=out, act="silu", out=out)
    assert torch.equal(first[before: n - behind], out[before: n - behind])


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (3, 1)])
def test_gradient(il, case, dtype, pad, shift):
    sizes, before, behind, k, m = CASES[case]
    G, n = len(sizes), before + sum(sizes) + behind
    gen = _gen(case + 17 * pad)
    X, W = _matrix(n, k, dtype, gen, pad, shift), _matrices(G, k, m, dtype, gen, pad, shift, 1 / math.sqrt(k))
    D, Z, dX = (_matrix(n, c, dtype, gen, pad, shift, s) for c, s in ((m, 1.0), (m, 2.0), (k, 1.0)))
    dW, db = _matrices(G, k, m, dtype, gen, pad, shift), _matrix(G, m, dtype, gen, pad, shift)
    offsets = _offsets(sizes, before)
    at = offsets.tolist()
    for t in (X, D, Z):
        if before:
            t[:before] = float("nan")
        if behind:
            t[n - behind:] = float("nan")
    ug = U[dtype] if dtype == BF16 else 0.0
    for act in ACTS:
        old = dX.clone()
        got = il.ilargi_grouped_linear_grad(D, X, W, offsets, pre=Z if act != "none" else None, act=act, d_X=dX, d_W=dW, d_bias=db)
        assert got[0] is dX and got[1] is dW and got[2] is db
        for g in range(G):
            s = slice(at[g], at[g + 1])
            x, w, d = X[s].double(), W[g].double(), D[s].double()
            grad, slack, rows = d * _slope(Z[s].double(), act), (0.0 if act == "none" else 32 * E), at[g + 1] - at[g]
            for res, want, size, raw, r, rounded in (
                    (dX[s], grad @ w.t(), grad.abs() @ w.t().abs(), d.abs() @ w.t().abs(), m, ug),
                    (dW[g], x.t() @ grad, x.t().abs() @ grad.abs(), x.t().abs() @ d.abs(), rows, ug),
                    (db[g], grad.sum(0), grad.abs().sum(0), d.abs().sum(0), rows, 0.0)):
                err = size * ((rounded if act != "none" else 0.0) + (r + 4) * E) * 1.01 + 1.01 * slack * raw
                _within(res, want, err, dtype, (act, g, rows))
            if rows == 0:
                assert bool((dW[g] == 0).all()) and bool((db[g] == 0).all())
        assert torch.equal(torch.nan_to_num(dX[:before]), torch.nan_to_num(old[:before])) and torch.equal(dX[n - behind:], old[n - behind:])
    # added to what is there; parts that are not asked for; the same bits again
    add_W, add_b = dW.clone(), db.clone()
    one = il.ilargi_grouped_linear_grad(D, X, W, offsets, pre=Z, act="gelu", d_X=None, d_W=add_W, d_bias=add_b, accumulate=True)
    assert one[0] is None
    for got, base in ((add_W, dW), (add_b, db)):
        # twice the stored value: the sum before its rounding is within u of it, and rounds once more
        assert bool(((got.double() - 2 * base.double()).abs() <= 2.02 * U[dtype] * (2 * base.double().abs())  + 1e-37).all())
    only = il.ilargi_grouped_linear_grad(D, X, W, offsets, pre=Z, act="gelu", d_W=None, d_bias=None)
    assert only[1] is None and only[2] is None and torch.equal(only[0][before: n - behind], dX[before: n - behind])
    assert torch.equal(il.ilargi_grouped_linear_grad(D, X, W, offsets, pre=Z, act="gelu", d_X=None, d_W=None)[2], db)
    assert torch.equal(il.ilargi_grouped_linear_grad(D, X, W, offsets, pre=Z, act="gelu", d_X=None, d_bias=None)[1], dW)
    again = il.ilargi_grouped_linear_grad(D, X, W, offsets, pre=Z, act="gelu")
    assert torch.equal(again[0][before: n - behind], dX[before: n - behind]) and torch.equal(again[1], dW) and torch.equal(again[2], db)


# enough work for the largest blocks and parts of long groups, and for operands that are laid out first
LARGE = [([700, 20, 1300], 512, 768), ([2100, 1], 520, 1016), ([40, 2500, 0, 700], 301, 603), ([3000, 2000], 256, 128), ([1200, 900], 1024, 1031)]


@pytest.mark.parametrize("case", range(len(LARGE)))
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (3, 1)])
def test_large(il, case, dtype, pad, shift):
    CASES.append((LARGE[case][0], 2, 3, *LARGE[case][1:]))
    try:
        test_forward(il, len(CASES) - 1, dtype, pad, shift)
        test_gradient(il, len(CASES) - 1, dtype, pad, shift)
    finally:
        CASES.pop()


def test_many_groups(il):
    """More groups than are sorted by size, and than one turn of the index takes."""
    gen = _gen(7)
    for dtype in (F32, BF16):
        for G in (513, 1024, 2500):
            sizes = torch.randint(0, 4, (G,), generator=gen, device="cuda")
            sizes[G // 2] = 400
            offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), sizes.cumsum(0)]).int()
            n, k, m = int(offsets[-1]) + 2, 16, 24
            X, W, D = _matrix(n, k, dtype, gen), _matrices(G, k, m, dtype, gen), _matrix(n, m, dtype, gen)
            ids = torch.repeat_interleave(torch.arange(G, device="cuda"), sizes)
            out = il.ilargi_grouped_linear(X, W, offsets)
            want = (X[:-2].double()[:, :, None] * W.double()[ids]).sum(1)
            size = (X[:-2].double()[:, :, None] * W.double()[ids]).abs().sum(1)
            _within(out[:-2], want, (k + 3) * E * size, dtype, "out")
            dX, dW, db = il.ilargi_grouped_linear_grad(D, X, W, offsets)
            prod = X[:-2].double()[:, :, None] * D[:-2].double()[:, None, :]
            into = lambda t: torch.zeros(G, *t.shape[1:], dtype=torch.float64, device="cuda").index_add_(0, ids, t)
            _within(dW, into(prod), 404 * E * into(prod.abs()), dtype, "dW")
            _within(db, into(D[:-2].double()), 404 * E * into(D[:-2].double().abs()), dtype, "db")
            t = D[:-2].double()[:, None, :] * W.double()[ids]
            _within(dX[:-2], t.sum(2), (m + 4) * E * t.abs().sum(2), dtype, "dX")


def test_offsets_that_are_not_ascending(il):
    """They count as the nearest that are: no row is read or written twice, none outside the matrices."""
    gen = _gen(4)
    n, k, m = 50, 24, 40
    for dtype in (F32, BF16):
        X, W, D = _matrix(n, k, dtype, gen), _matrices(5, k, m, dtype, gen), _matrix(n, m, dtype, gen)
        bad = torch.tensor([-7, 10, 4, 30, 2 ** 31 - 1, 20], dtype=torch.int32, device="cuda")
        good = torch.tensor([0, 10, 10, 30, 50, 50], dtype=torch.int32, device="cuda")
        assert torch.equal(il.ilargi_grouped_linear(X, W, bad), il.ilargi_grouped_linear(X, W, good))
        for a, b in zip(il.ilargi_grouped_linear_grad(D, X, W, bad), il.ilargi_grouped_linear_grad(D, X, W, good)):
            assert torch.equal(a, b)


def test_no_rows_and_no_groups(il):
    for dtype in (F32, BF16):
        X, W = torch.empty(0, 16, dtype=dtype, device="cuda"), torch.ones(3, 16, 8, dtype=dtype, device="cuda")
        offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
        assert il.ilargi_grouped_linear(X, W, offsets).shape == (0, 8)
        D = torch.empty(0, 8, dtype=dtype, device="cuda")
        dX, dW, db = il.ilargi_grouped_linear_grad(D, X, W, offsets)
        assert dX.shape == (0, 16) and bool((dW == 0).all()) and bool((db == 0).all())
        il.ilargi_grouped_linear_grad(D, X, W, offsets, d_X=None, d_W=dW.fill_(2), d_bias=db.fill_(3), accumulate=True)
        assert bool((dW == 2).all()) and bool((db == 3).all())
        Y = torch.ones(5, 16, dtype=dtype, device="cuda")
        out = torch.full((5, 8), 7.0, dtype=dtype, device="cuda")
        il.ilargi_grouped_linear(Y, W[:0], offsets[:1], out=out)
        il.ilargi_grouped_linear(Y, W, offsets, out=out)
        assert bool((out == 7).all())


def test_workspace_is_enough_and_no_more_is_touched(il):
    gen = _gen(21)
    for dtype in (F32, BF16):
        for sizes, k, m in (([1, 1], 4099, 70), ([5, 0, 300], 512, 512), ([9] * 7, 40, 24), ([1500, 700], 601, 701), ([2000], 24, 16), ([900, 40], 1024, 512)):
            n, G = sum(sizes) + 3, len(sizes)
            X, W, D, Z = _matrix(n, k, dtype, gen), _matrices(G, k, m, dtype, gen, scale=0.05), _matrix(n, m, dtype, gen), _matrix(n, m, dtype, gen)
            offsets = _offsets(sizes, 1)
            for which, nbytes in enumerate(il.ilargi_grouped_linear_workspace_bytes(G, n, k, m, dtype)):
                store = torch.full((nbytes + 512,), 171, dtype=torch.uint8, device="cuda")
                ws = store[256: 256 + nbytes]
                if which == 0:
                    got, want = ([il.ilargi_grouped_linear(X, W, offsets, act="gelu", workspace=w)] for w in (ws, None))
                else:
                    got, want = (il.ilargi_grouped_linear_grad(D, X, W, offsets, pre=Z, act="silu", workspace=w) for w in (ws, None))
                assert all(torch.equal(a, b) for a, b in zip(got, want))
                assert bool((store[:256] == 171).all()) and bool((store[256 + nbytes:] == 171).all())


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(il, act):
    """L = sum(Y o layers(X, W, b)): central differences of L in 64 bits along random directions against the kernels' gradients, as for
    one layer: off by h^2 / 6 of the third derivative.  Where relu's z changes its sign between the two ends (or is not on the side that
    float32 found), the difference quotient of an entry lies between 0 and its |dz|, and its gradient is one of the two: off by at most |Y| |dz|,
    which is added up over those entries."""
    gen = _gen(11)
    sizes, k, m, h = [60, 0, 1, 89], 36, 44, 1e-5
    n, offsets = sum(sizes), _offsets(sizes, 0)
    at = offsets.tolist()
    X, W, b = (torch.randn(s, generator=gen, device="cuda") for s in ((n, k), (4, k, m), (4, m)))
    W /= 6
    Y = torch.randn(n, m, generator=gen, device="cuda")
    pre = torch.empty(n, m, device="cuda")
    il.ilargi_grouped_linear(X, W, offsets, bias=b, act=act, pre=pre)
    grads = il.ilargi_grouped_linear_grad(Y, X, W, offsets, pre=pre, act=act)
    Z = lambda x, w, c: torch.cat([x[at[g]: at[g + 1]] @ w[g] + c[g] for g in range(4)])
    L = lambda z: float((Y.double() * _f(z, act)).sum())
    ops = [X.double(), W.double(), b.double()]
    for q, grad in enumerate(grads):
        v = torch.randn(grad.shape, generator=gen, device="cuda").double()
        up, down = ([o + s * h * v if i == q else o for i, o in enumerate(ops)] for s in (1, -1))
        z_up, z_down = Z(*up), Z(*down)
        numeric, parts = (L(z_up) - L(z_down)) / (2 * h), grad.double() * v
        tol = 1e-5 * float(parts.abs().sum())
        if act == "relu":
            kinks = ((z_up > 0) != (z_down > 0)) | ((z_up > 0) != (pre > 0))
            assert int(kinks.sum()) < 20
            tol += float((Y.double() * (z_up - z_down) / (2 * h)).abs()[kinks].sum())
        assert abs(numeric - float(parts.sum())) <= tol


def test_values_that_are_not_finite(il):
    """A row that holds NaN spoils itself; a matrix that does, its own group."""
    gen = _gen(4)
    for dtype in (F32, BF16):
        for sizes, k, m in (([3, 4], 64, 32), ([130, 200, 70], 96, 144)):
            n, G = sum(sizes), len(sizes)
            X, W, offsets = _matrix(n, k, dtype, gen), _matrices(G, k, m, dtype, gen), _offsets(sizes, 0)
            X[1, k // 3] = float("nan")
            bad = torch.isnan(il.ilargi_grouped_linear(X, W, offsets)).any(1)
            assert bool(bad[1]) and int(bad.sum()) == 1
            X[1, k // 3] = 0.0
            W[1, 0, 0] = float("inf")
            bad = (~torch.isfinite(il.ilargi_grouped_linear(X, W, offsets))).any(1)
            assert not bool(bad[: sizes[0]].any()) and bool(bad[sizes[0]: sizes[0] + sizes[1]].all()) and not bool(bad[sizes[0] + sizes[1]:].any())
            D = _matrix(n, m, dtype, gen)
            D[n - 1] = float("nan")
            dX, dW, db = il.ilargi_grouped_linear_grad(D, X, W[:, :, :].clone().nan_to_num(posinf=1.0), offsets)
            assert bool(torch.isfinite(dW[:-1]).all()) and bool(torch.isnan(dW[-1]).all()) and bool(torch.isfinite(db[:-1]).all()) and int(torch.isnan(dX).any(1).sum()) == 1


def test_on_another_stream_and_in_a_graph(il):
    gen = _gen(12)
    for dtype, sizes, k, m in ((F32, [40, 0, 56], 200, 136), (BF16, [300, 20], 200, 136), (BF16, [2, 1, 0], 512, 256)):
        n, G = sum(sizes), len(sizes)
        X, W, D, b = _matrix(n, k, dtype, gen), _matrices(G, k, m, dtype, gen, scale=0.1), _matrix(n, m, dtype, gen), _matrix(G, m, dtype, gen)
        offsets = _offsets(sizes, 0)
        out, pre, dX, dW, db = torch.empty_like(D), torch.empty_like(D), torch.empty_like(X), torch.empty_like(W), torch.empty_like(b)
        ws = torch.empty(max(il.ilargi_grouped_linear_workspace_bytes(G, n, k, m, dtype)), dtype=torch.uint8, device="cuda")
        all_of = (out, pre, dX, dW, db)

        def step(stream=None):
            il.ilargi_grouped_linear(X, W, offsets, bias=b, act="gelu", out=out, pre=pre, workspace=ws, stream=stream)
            il.ilargi_grouped_linear_grad(D, X, W, offsets, pre=pre, act="gelu", d_X=dX, d_W=dW, d_bias=db, workspace=ws, stream=stream)

        step()
        want = [t.clone() for t in all_of]
        side = torch.cuda.Stream()
        for t in all_of:
            t.zero_()
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        side.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, all_of))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for q in range(3):
            X.copy_(torch.randn(n, k, generator=gen, device="cuda"))
            offsets[1] = max(0, int(offsets[1]) - 1)               # other groups in the same graph
            step()
            want = [t.clone() for t in all_of]
            for t in all_of:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(want, all_of))


def test_groups_of_a_join(il):
    """The inverse index of a plan says which rows join which: each row of the joined table has a layer of its own."""
    import datagen
    rng = datagen.rng_for(3)
    schema = datagen.star_schema(rng, 3000, 6, [(20, 5, ("zipf", 1.1))])
    sources = il.schema_to_device(schema)
    plan = il.ilargi_plan_create(sources, schema.r_T, schema.c_T)
    rowptr, perm = (torch.from_numpy(v).cuda() for v in il.ilargi_plan_inverse_index(plan, 1))
    T = il.ilargi_materialize(plan)
    gen = _gen(1)
    W, b = _matrices(20, schema.c_T, 8, F32, gen), _matrix(20, 8, F32, gen)
    rows = il.ilargi_embed(T, perm)
    out = torch.empty(schema.r_T, 8, device="cuda")
    out[perm.long()] = il.ilargi_grouped_linear(rows, W, rowptr, bias=b, act="relu")
    fk = torch.as_tensor(schema.sources[1].row_idx, device="cuda").long()
    prod = T.double()[:, :, None] * W.double()[fk]
    want = (prod.sum(1) + b.double()[fk]).clamp(min=0)
    _within(out, want, (schema.c_T + 3) * E * (prod.abs().sum(1) + b.double().abs()[fk]), F32, "join")


def test_python_refuses(il):
    X, W, o = torch.zeros(4, 6, device="cuda"), torch.zeros(3, 6, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: il.ilargi_grouped_linear(X, W[:, :5], o), lambda: il.ilargi_grouped_linear(X, W, o[:3]), lambda: il.ilargi_grouped_linear(X, W[0], o),
                 lambda: il.ilargi_grouped_linear(X, W, o, act="tanh"), lambda: il.ilargi_grouped_linear(X, W, o, out=torch.zeros(4, 7, device="cuda")),
                 lambda: il.ilargi_grouped_linear_grad(X, X, W, o), lambda: il.ilargi_grouped_linear_grad(torch.zeros(4, 8, device="cuda"), X, W, o, act="relu"),
                 lambda: il.ilargi_grouped_linear_grad(torch.zeros(4, 8, device="cuda"), X, W, o, accumulate=True)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: il.ilargi_grouped_linear(X, W.bfloat16(), o), lambda: il.ilargi_grouped_linear(X, W, o.long()), lambda: il.ilargi_grouped_linear(X, W.transpose(1, 2).contiguous().transpose(1, 2), o),
                 lambda: il.ilargi_grouped_linear(X, W[:1].expand(3, 6, 8), o)):
        with pytest.raises(TypeError):
            call()
