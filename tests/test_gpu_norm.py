"""Norms around a residual sum and their gradients against 64 bits.

Bounds, with E = 2^-24 and u half a step of the layer's type (2^-24, 2^-8).  A row of m columns is summed by at most
m / 64 + 12 additions in a row and a tree, so a sum of m terms is off by at most (m / 64 + 14) E of the sum of their sizes; S below is
(m / 32 + 40) E, which covers a mean, the variance around it, the reciprocal root and the products that follow.  (A thread holds at most
16 values of a row, a wavefront adds 64 threads in 6 steps, 16 wavefronts are added in a row.)

forward: |N(v)| is off by S (|v^| + mean|v| / dev [centred: what the mean loses] ) |gain| + E |bias|, and by the error of v itself times
(1 + |v^| mean|v^|) / dev |gain|.  The gate's activation is good to 16 E (1 + |z|), its slope to 32 E (1 + |z|).
gradient: the same rules for t: dv = by (t - v^ mean(t v^) - mean(t)); errors of t and of v^ go through it with at most
by (|e| + |v^| mean|e v^| + mean|e|).  They are propagated with the formulas below, in 64 bits, entry by entry (`Err`).
Sums over rows: n terms in at most n + 20 additions, (n + 24) E of the sum of sizes, and the errors of the terms.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
E = 2.0 ** -24
EPS = 1e-6


@pytest.fixture(scope="module")
def il():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_01985_amd as mod
    return mod


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _matrix(rows, cols, dtype, gen, pad=0, shift=0, scale=1.0, add=0.0):
    store = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    m = store[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=gen, device="cuda") * scale + add)
    return m


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


class Norm:
    """v normalised in 64 bits, with bounds on what float32 loses: `unit`, `err` of it, `by`."""

    def __init__(self, v, err, kind):
        m = v.shape[1]
        self.kind, self.S = kind, (m / 32 + 40) * E
        mean = lambda t: t.mean(1, keepdim=True)
        if kind == "none":
            self.unit, self.err, self.by = v, err, torch.ones(v.shape[0], 1, dtype=torch.float64, device=v.device)
            return
        c = v - mean(v) if kind == "centred" else v
        ec = err + (mean(err) + self.S * mean(v.abs()) + E * v.abs() if kind == "centred" else 0.0)
        self.by = 1.0 / torch.sqrt(mean(c * c) + EPS)
        self.unit = c * self.by
        rel = (self.by ** 2) * mean(c.abs() * ec + 0.5 * ec * ec) + self.S
        self.err = self.by * ec + self.unit.abs() * rel + E * self.unit.abs()
        self.rel = rel

    def back(self, t, et):
        """The gradient before the norm for t behind it, and its bound."""
        if self.kind == "none":
            return t, et
        mean = lambda s: s.mean(1, keepdim=True)
        along = mean(t * self.unit)
        ea = mean(et * self.unit.abs() + t.abs() * self.err + et * self.err) + self.S * mean((t * self.unit).abs())
        out = t - self.unit * along
        eo = et + self.unit.abs() * ea + self.err * (along.abs() + ea)
        size = t.abs() + (self.unit * along).abs()
        if self.kind == "centred":
            out = out - mean(t)
            eo = eo + mean(et) + self.S * mean(t.abs())
            size = size + mean(t.abs())
        return self.by * out, self.by * (1 + self.rel) * (eo + 6 * E * size) + self.by * out.abs() * self.rel


def _oracle(case, h, x, gate, g1, b1, g2, b2, act, scale, dr=None, dy=None):
    """Every result with its bound before it is rounded to its type."""
    first, second = case
    d = lambda t: t.double() if t is not None else None
    h, x, gate, g1, b1, g2, b2, dr, dy = map(d, (h, x, gate, g1, b1, g2, b2, dr, dy))
    one = torch.ones((), dtype=torch.float64, device=h.device)
    n1 = Norm(h, torch.zeros_like(h), first)
    u = n1.unit * (g1 if g1 is not None else one) + (b1 if b1 is not None else 0.0)
    eu = n1.err * (g1.abs() if g1 is not None else one) + 2 * E * (u.abs() + (b1.abs() if b1 is not None else 0.0))
    f, ef = (one, 0.0) if gate is None else (_f(gate, act), 0.0 if act == "none" else 16 * E * (1 + gate.abs()))
    v = scale * f * u
    ev = abs(scale) * ((f.abs() + ef) * eu + ef * u.abs()) + 3 * E * v.abs()
    r = v + (x if x is not None else 0.0)
    er = ev + E * r.abs() + E * v.abs()
    n2 = Norm(r, er, second)
    out = {"r": (r, er)}
    if second != "none":
        y = n2.unit * (g2 if g2 is not None else one) + (b2 if b2 is not None else 0.0)
        out["y"] = (y, n2.err * (g2.abs() if g2 is not None else one) + 2 * E * (y.abs() + (b2.abs() if b2 is not None else 0.0)))
    if dr is None and dy is None:
        return out
    n = h.shape[0]
    over_rows = lambda t, et: (t.sum(0), (et + (n + 24) * E * (t.abs() + et)).sum(0))
    t, et = (dr, torch.zeros_like(dr)) if dr is not None else (torch.zeros_like(h), torch.zeros_like(h))
    if second != "none":
        dy = dy if dy is not None else torch.zeros_like(h)
        out["d_gain2"] = over_rows(dy * n2.unit, dy.abs() * n2.err + E * (dy * n2.unit).abs())
        out["d_bias2"] = over_rows(dy, torch.zeros_like(dy))
        b, eb = n2.back(dy * (g2 if g2 is not None else one), E * (dy * (g2 if g2 is not None else one)).abs())
        t, et = t + b, eb + E * (t.abs() + b.abs())
    out["d_x"] = (t, et)
    t, et = scale * t, abs(scale) * et + 2 * E * (scale * t).abs()
    if gate is not None:
        s, es = _slope(gate, act), 0.0 if act == "none" else 32 * E * (1 + gate.abs())
        g = s * u * t
        out["d_gate"] = (g, (s.abs() + es) * ((u.abs() + eu) * et + eu * t.abs()) + es * (u * t).abs() + 3 * E * g.abs())
        if gate.dim() == 1:
            out["d_gate"] = over_rows(*out["d_gate"])
    t, et = t * f, (f.abs() + ef) * et + ef * t.abs() + E * (t * f).abs()
    out["d_gain1"] = over_rows(t * n1.unit, t.abs() * n1.err + et * (n1.unit.abs() + n1.err) + E * (t * n1.unit).abs())
    out["d_bias1"] = over_rows(t, et)
    g = g1 if g1 is not None else one
    out["d_h"] = n1.back(t * g, et * g.abs() + E * (t * g).abs())
    return out


def _close(got, bound, dtype, name):
    want, err = bound
    err = 1.01 * err + 1e-37
    off = (got.double() - want).abs() - (err + U[dtype] * (want.abs() + err))
    assert bool((off <= 0).all()), (name, float(off.max()), float(want.abs().max()))


GRADS = ("d_h", "d_x", "d_gate", "d_gain1", "d_bias1", "d_gain2", "d_bias2")
# rows, columns: single ones, shorter than a piece, odd, every number of threads a row, the most columns
SHAPES = [(0, 5), (1, 1), (3, 2), (2, 7), (5, 8), (1, 64), (9, 65), (33, 127), (17, 128), (40, 220), (130, 333), (7, 513), (65, 1000), (4, 1025), (3, 2049), (300, 96),
          (5, 4096), (2, 4103), (3, 8192), (2, 9001), (1, 16384)]
KINDS = [("rms", "rms"), ("centred", "none"), ("none", "centred"), ("rms", "none"), ("none", "none"), ("centred", "centred")]


@pytest.mark.parametrize("n,m", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (3, 1)])
def test_forward_and_gradient(il, n, m, dtype, pad, shift):
    gen = _gen(n + 3 * m + pad)
    mat = lambda scale=1.0, add=0.0: _matrix(n, m, dtype, gen, pad, shift, scale, add)
    vec = lambda scale=1.0, add=0.0: (torch.randn(m, generator=gen, device="cuda") * scale + add).to(dtype)
    h, x, gates, dr, dy = mat(2.0, 0.5), mat(3.0), mat(), mat(0.01), mat(0.01)
    g1, b1, row, g2, b2 = vec(0.2, 1.0), vec(0.1), vec(0.5), vec(0.2, 1.0), vec(0.1)
    r, y, dh, dx, dg = (mat() for _ in range(5))
    for q, (first, second) in enumerate(KINDS):
        act = ["none", "sigmoid", "silu", "relu", "gelu", "silu"][q]
        gate = [row, gates, gates, None, row, gates][q]
        args = dict(first=first, gain1=g1 if q != 3 else None, bias1=b1 if q % 2 else None, gate=gate, gate_act=act, scale=0.7 - 0.3 * q, x=x if q != 2 else None,
                    second=second, gain2=g2 if second != "none" and q != 5 else None, bias2=b2 if second == "centred" else None, eps=EPS)
        y_in = dy if second != "none" else None
        want = _oracle((first, second), h, args["x"], gate, args["gain1"], args["bias1"], args["gain2"], args["bias2"], act, args["scale"], dr, y_in)
        got = il.ilargi_norm(h, r=r, y=y if second != "none" else None, **args)
        assert got[0] is r
        _close(r, want["r"], dtype, "r")
        if second != "none":
            _close(y, want["y"], dtype, "y")
        filled = dict(d_h=dh, d_x=dx, d_gate=dg if gate is gates else (torch.empty_like(row) if gate is row else None), d_gain1=torch.empty_like(row), d_bias1=torch.empty_like(row),
                      d_gain2=torch.empty_like(row) if second != "none" else None, d_bias2=torch.empty_like(row) if second != "none" else None)
        back = il.ilargi_norm_grad(dr, y_in, h, **args, **filled)
        for name, t in zip(GRADS, back):
            assert t is filled[name]
            if t is not None:
                _close(t, want[name], dtype, (name, first, second))
        # the same bits again, in new tensors; what has no operand is not made
        again = dict(zip(GRADS, il.ilargi_norm_grad(dr, y_in, h, **args)))
        made = dict(d_h=True, d_x=args["x"] is not None, d_gate=gate is not None, d_gain1=args["gain1"] is not None, d_bias1=args["bias1"] is not None,
                    d_gain2=args["gain2"] is not None, d_bias2=args["bias2"] is not None)
        for name in GRADS:
            assert (again[name] is not None) == made[name]
            assert again[name] is None or torch.equal(again[name], filled[name])


def test_long_sums_over_rows(il):
    """Many rows a workgroup, and the sums added to what is there."""
    gen = _gen(5)
    for dtype, n, m in ((F32, 70_001, 5), (BF16, 30_011, 40), (F32, 5000, 700), (BF16, 2051, 1030)):
        h, x, gate, dr, dy = (_matrix(n, m, dtype, gen) for _ in range(5))
        row = gate[0].clone()
        args = dict(first="rms", gain1=row, gate=row, gate_act="silu", x=x, second="centred", bias2=row, scale=0.5)
        want = _oracle(("rms", "centred"), h, x, row, row, None, None, row, "silu", 0.5, dr, dy)
        got = dict(zip(GRADS, il.ilargi_norm_grad(dr, dy, h, d_gain2=torch.empty_like(row), d_bias1=torch.empty_like(row), **args)))
        sums = [k for k in GRADS if k not in ("d_h", "d_x")]
        for name in GRADS:
            _close(got[name], want[name], dtype, name)
        old = {k: torch.randn(m, generator=gen, device="cuda").to(dtype) for k in sums}
        into = {k: v.clone() for k, v in old.items()}
        il.ilargi_norm_grad(dr, dy, h, d_h=None, d_x=None, accumulate=True, **into, **args)
        for k in sums:
            w, e = want[k]
            _close(into[k], (w + old[k].double(), e + E * (w.abs() + old[k].double().abs())), dtype, k)


@pytest.mark.parametrize("kinds", [(a, b) for a in ("none", "rms", "centred") for b in ("none", "rms", "centred")])
@pytest.mark.parametrize("act", ["none", "sigmoid", "gelu"])
def test_every_pair_of_norms_where_rows_do_not_fill_their_threads(il, kinds, act):
    """Threads that hold no columns of a row, or columns that their neighbours have too, add nothing to its means: with a gate whose value
    at 0 is not 0, and without one."""
    gen = _gen(14)
    for dtype, n, m in ((F32, 40, 23), (F32, 9, 2369), (BF16, 30, 9), (BF16, 7, 1100)):
        h, x, dr, dy = (_matrix(n, m, dtype, gen) for _ in range(4))
        second = kinds[1] != "none"
        for gate in (None, h[0].clone(), x):
            args = dict(first=kinds[0], second=kinds[1], gate=gate, gate_act=act, x=x, scale=0.8)
            want = _oracle(kinds, h, x, gate, None, None, None, None, act, 0.8, dr, dy if second else None)
            for name, t in zip(("r", "y"), il.ilargi_norm(h, **args)):
                if t is not None:
                    _close(t, want[name], dtype, name)
            more = dict(d_gain1=torch.empty_like(h[0]), d_bias1=torch.empty_like(h[0]))
            for name, t in zip(GRADS, il.ilargi_norm_grad(dr, dy if second else None, h, **args, **more)):
                if t is not None:
                    _close(t, want[name], dtype, (name, gate is None))


def test_no_rows(il):
    e = torch.empty(0, 12, device="cuda")
    v = torch.ones(12, device="cuda")
    r, y = il.ilargi_norm(e, x=e, second="rms")
    assert r.shape == y.shape == (0, 12)
    got = dict(zip(GRADS, il.ilargi_norm_grad(e, e, e, gain1=v, gate=v, x=e, second="rms", gain2=v)))
    assert all(bool((got[k] == 0).all()) for k in ("d_gate", "d_gain1", "d_gain2"))
    kept = torch.full((12,), 3.0, device="cuda")
    il.ilargi_norm_grad(e, None, e, gain1=v, d_h=None, d_gain1=kept, accumulate=True)
    assert bool((kept == 3).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m", [(37, 333), (9, 4100), (5, 3), (700, 64)])
def test_in_place(il, dtype, n, m):
    gen = _gen(m)
    h, x, dr, dy, gate = (_matrix(n, m, dtype, gen, 3, 1) for _ in range(5))
    for kinds in (("rms", "centred"), ("none", "none")):
        args = dict(first=kinds[0], second=kinds[1], gate=gate, gate_act="sigmoid")
        second = kinds[1] != "none"
        r, y = il.ilargi_norm(h, x=x, **args)
        h2, x2 = h.clone(), x.clone()
        got = il.ilargi_norm(h2, x=x2, r=x2, y=h2 if second else None, **args)
        assert got[0] is x2 and torch.equal(x2, r) and (not second or torch.equal(h2, y))
        h3 = h.clone()
        assert torch.equal(il.ilargi_norm(h3, x=x, r=h3, y=None, **args)[0], r)
        want = il.ilargi_norm_grad(dr, dy if second else None, h, x=x, **args)
        dr2, dy2 = dr.clone(), dy.clone()
        il.ilargi_norm_grad(dr2, dy2 if second else None, h, x=x, d_x=dr2, d_h=dy2, **args)
        assert torch.equal(dr2, want[1]) and torch.equal(dy2, want[0])


def test_parts_that_are_not_wanted(il):
    gen = _gen(3)
    n, m = 50, 200
    h, x, gate, dr, dy = (_matrix(n, m, F32, gen) for _ in range(5))
    g = gate[0].clone()
    args = dict(first="rms", gain1=g, gate=gate, gate_act="silu", x=x, second="rms", gain2=g)
    whole = dict(zip(GRADS, il.ilargi_norm_grad(dr, dy, h, **args)))
    for name in ("d_h", "d_x", "d_gate", "d_gain1", "d_gain2"):
        only = dict(zip(GRADS, il.ilargi_norm_grad(dr, dy, h, **args, **{k: None for k in whole if k != name})))
        assert torch.equal(only[name], whole[name]) and all(only[k] is None for k in GRADS if k != name)
    r, y = il.ilargi_norm(h, **args)
    only_y = il.ilargi_norm(h, r=None, **args)
    assert only_y[0] is None and torch.equal(only_y[1], y)
    assert torch.equal(il.ilargi_norm(h, y=None, **args)[0], r)
    # gradients of one of the results
    zero = torch.zeros_like(dr)
    for a, b in (((dr, None), (dr, zero)), ((None, dy), (zero, dy))):
        for p, q in zip(il.ilargi_norm_grad(*a, h, **args), il.ilargi_norm_grad(*b, h, **args)):
            assert (p is None) == (q is None) and (p is None or torch.equal(p, q))


def test_workspace_is_enough_and_no_more_is_touched(il):
    gen = _gen(8)
    for dtype in (F32, BF16):
        for n, m in ((1, 5), (40, 40), (1500, 200), (700, 5000)):
            h, x, dr, dy = (_matrix(n, m, dtype, gen) for _ in range(4))
            g = h[0].clone()
            args = dict(gain1=g, bias1=g, gate=g, x=x, second="centred", gain2=g, bias2=g)
            nbytes = il.ilargi_norm_grad_workspace_bytes(n, m, dtype)
            store = torch.full((nbytes + 512,), 171, dtype=torch.uint8, device="cuda")
            got = il.ilargi_norm_grad(dr, dy, h, workspace=store[256: 256 + nbytes], **args)
            assert all(torch.equal(a, b) for a, b in zip(got, il.ilargi_norm_grad(dr, dy, h, **args)))
            assert bool((store[:256] == 171).all()) and bool((store[256 + nbytes:] == 171).all())


def test_values_that_are_not_finite_and_rows_of_zeros(il):
    gen = _gen(2)
    for dtype in (F32, BF16):
        for n, m in ((6, 40), (11, 333), (9, 2500)):
            h, x = _matrix(n, m, dtype, gen), _matrix(n, m, dtype, gen)
            h[1] = 0.0
            h[3, m // 2] = float("nan")
            h[4, m - 1] = float("inf")
            for kind in ("rms", "centred"):
                r, y = il.ilargi_norm(h, first=kind, x=x, second="rms")
                assert torch.equal(r[1], x[1])                         # nothing over the root of eps
                bad = ~torch.isfinite(y).all(1)
                assert [int(q) for q in bad.nonzero()] == [3, 4]
                good = il.ilargi_norm(h[[0, 1, 2, 5]], first=kind, x=x[[0, 1, 2, 5]], second="rms")
                assert torch.equal(good[0], r[[0, 1, 2, 5]]) and torch.equal(good[1], y[[0, 1, 2, 5]])
    # a mean far from the deviations around it
    h = torch.randn(50, 700, generator=gen, device="cuda") + 1000.0
    r, _ = il.ilargi_norm(h, first="centred")
    _close(r, _oracle(("centred", "none"), h, None, None, None, None, None, None, "none", 1.0)["r"], F32, "r")


def test_gradient_against_differences(il):
    """L = sum(A o r + B o y): central differences of L in 64 bits along random directions.  They are off by h^2 / 6 of the third
    derivative, below 1e-7 of L here; the gradients by float32's rounding."""
    gen = _gen(13)
    n, m, h0 = 20, 60, 1e-5
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    for first, second, row in (("rms", "centred", False), ("centred", "rms", True)):
        ops = dict(h=new(n, m), x=new(n, m), gate=new(m) if row else new(n, m), gain1=new(m), bias1=new(m), gain2=new(m), bias2=new(m))
        A, B = new(n, m), new(n, m)
        names = dict(h="d_h", x="d_x", gate="d_gate", gain1="d_gain1", bias1="d_bias1", gain2="d_gain2", bias2="d_bias2")
        got = dict(zip(GRADS, il.ilargi_norm_grad(A, B, ops["h"], first=first, second=second, gate_act="silu", scale=0.6, **{k: v for k, v in ops.items() if k != "h"})))

        def L(o):
            w = _oracle((first, second), o["h"], o["x"], o["gate"], o["gain1"], o["bias1"], o["gain2"], o["bias2"], "silu", 0.6)
            return float((A.double() * w["r"][0]).sum() + (B.double() * w["y"][0]).sum())

        base = {k: v.double() for k, v in ops.items()}
        for k in ops:
            v = torch.randn(ops[k].shape, generator=gen, device="cuda").double()
            numeric = (L({**base, k: base[k] + h0 * v}) - L({**base, k: base[k] - h0 * v})) / (2 * h0)
            parts = got[names[k]].double() * v
            assert abs(numeric - float(parts.sum())) <= 1e-5 * float(parts.abs().sum()), k


def test_on_another_stream_and_in_a_graph(il):
    gen = _gen(12)
    for dtype, n, m in ((F32, 90, 333), (BF16, 33, 4096)):
        h, x, gate, dr, dy = (_matrix(n, m, dtype, gen) for _ in range(5))
        g = h[0].clone()
        args = dict(gain1=g, gate=gate, gate_act="silu", x=x, second="rms", gain2=g)
        r, y = torch.empty_like(x), torch.empty_like(x)
        out = dict(d_h=torch.empty_like(x), d_x=torch.empty_like(x), d_gate=torch.empty_like(x), d_gain1=torch.empty_like(g), d_gain2=torch.empty_like(g))
        ws = torch.empty(il.ilargi_norm_grad_workspace_bytes(n, m, dtype), dtype=torch.uint8, device="cuda")
        all_of = lambda: [r, y, *out.values()]

        def step(stream=None):
            il.ilargi_norm(h, r=r, y=y, stream=stream, **args)
            il.ilargi_norm_grad(dr, dy, h, workspace=ws, stream=stream, **args, **out)

        step()
        want = [t.clone() for t in all_of()]
        side = torch.cuda.Stream()
        for t in all_of():
            t.zero_()
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, all_of()))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(3):
            h.copy_(torch.randn(n, m, generator=gen, device="cuda"))
            step()
            want = [t.clone() for t in all_of()]
            for t in all_of():
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, all_of()))


def test_no_gate_with_rows(il):
    """A block that says gate_rows and has no gate, as the C interface allows: as without."""
    import ctypes
    gen = _gen(7)
    n, m = 20, 100
    h, d = _matrix(n, m, F32, gen), _matrix(n, m, F32, gen)
    r, dh = torch.empty_like(h), torch.empty_like(h)
    block = il.NormStruct(n, m, 0, 1, 0, 3, 1, 0.5, EPS, h.data_ptr(), None, None, None, None, None, None, m, 0, 0)
    stream = torch.cuda.current_stream().cuda_stream
    assert il.lib.ilargi_norm(ctypes.byref(block), r.data_ptr(), m, None, 0, stream) == il.OK
    grads = il.NormGradsStruct(dh.data_ptr(), None, None, None, None, None, None, m, 0, 0)
    assert il.lib.ilargi_norm_grad(ctypes.byref(block), d.data_ptr(), m, None, 0, ctypes.byref(grads), 0, None, 0, stream) == il.OK
    assert torch.equal(r, il.ilargi_norm(h, scale=0.5, eps=EPS)[0]) and torch.equal(dh, il.ilargi_norm_grad(d, None, h, scale=0.5, eps=EPS)[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", [8192, 6001, 12_000])
def test_wide_rows_with_all_their_sums(il, dtype, m):
    """Rows whose sums do not fit the registers, eagerly and in a graph."""
    gen = _gen(m)
    n = 300
    h, x, dr, dy = (_matrix(n, m, dtype, gen) for _ in range(4))
    v = [torch.randn(m, generator=gen, device="cuda").to(dtype) for _ in range(5)]
    args = dict(first="centred", gain1=v[0], bias1=v[1], gate=v[2], gate_act="silu", x=x, second="centred", gain2=v[3], bias2=v[4])
    want = _oracle(("centred", "centred"), h, x, v[2], v[0], v[1], v[3], v[4], "silu", 1.0, dr, dy)
    out = {k: torch.empty(n, m, dtype=dtype, device="cuda") if k in ("d_h", "d_x") else torch.empty(m, dtype=dtype, device="cuda") for k in GRADS}
    ws = torch.empty(il.ilargi_norm_grad_workspace_bytes(n, m, dtype), dtype=torch.uint8, device="cuda")
    step = lambda: il.ilargi_norm_grad(dr, dy, h, workspace=ws, **args, **out)
    step()
    for k in GRADS:
        _close(out[k], want[k], dtype, k)
    kept = [out[k].clone() for k in GRADS]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for k in GRADS:
            out[k].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], t) for k, t in zip(GRADS, kept))


def test_python_refuses(il):
    a, v = torch.zeros(4, 8, device="cuda"), torch.zeros(8, device="cuda")
    bad = [lambda: il.ilargi_norm(a, first="layer"), lambda: il.ilargi_norm(a, x=a[:3]), lambda: il.ilargi_norm(a, gain1=v[:7]), lambda: il.ilargi_norm(a, gate_act="tanh"),
           lambda: il.ilargi_norm(a[0]), lambda: il.ilargi_norm_grad(a, None, a, gain1=v, accumulate=True)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: il.ilargi_norm(a, x=a.half()), lambda: il.ilargi_norm(a, gain1=v.bfloat16()), lambda: il.ilargi_norm(a.t()), lambda: il.ilargi_norm(a, r=torch.zeros(4, 8))):
        with pytest.raises((TypeError, ValueError)):
            call()
    for call in (lambda: il.ilargi_norm(a, y=a.clone()), lambda: il.ilargi_norm(a, gain2=v), lambda: il.ilargi_norm_grad(a, a, a)):
        with pytest.raises(il.IlargiError):
            call()
