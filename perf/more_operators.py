"""Operators of deeper models over a join, as measurable cases.

  norm          the end of a block: its output normalised, gated and added to the residual stream, and the stream normalised for
                the next block;  r = x + scale f(gate) o N1(h),  y = N2(r)
  norm_grad     its gradients
  grouped       a dense layer of its own for every group of rows:  f(X_g W_g + bias_g), groups of ragged sizes
  grouped_grad  its gradients
  clip          the norm over many tensors, and the tensors scaled to a largest norm

`run` computes each of them with elementary torch operations in 32 bits (`own` false) or through this package's entry
points (`own` true).  `exact` is the definition in 64 bits.

Every case has the element `type` ("f32" or "bf16") and `pad`, the columns that the caller's matrices have beyond the ones
used (the operands are then column slices of wider tensors).
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-6
GRAD = 1e-3           # size of a gradient's entries


def listed():
    return [
        # One joined row between two blocks of a served model: latency.
        {"name": "norm_one_row", "op": "norm", "n": 1, "m": 4096, "first": "rms", "second": "rms", "gate": "row", "act": "none", "stream": True, "type": "bf16", "pad": 0},
        # Joined rows with an odd number of columns, means subtracted, a gate for every entry.
        {"name": "norm_ragged", "op": "norm", "n": 10_007, "m": 333, "first": "centred", "second": "none", "gate": "rows", "act": "sigmoid", "stream": True, "type": "f32", "pad": 0},
        # A training batch: norms on both sides of the residual sum.
        {"name": "norm_train", "op": "norm", "n": 16_384, "m": 4096, "first": "rms", "second": "rms", "gate": "row", "act": "none", "stream": True, "type": "bf16", "pad": 0},
        # The gradient over 100,000 joined rows of 220 columns, a learned factor a column.
        {"name": "norm_grad_join", "op": "norm_grad", "n": 100_000, "m": 220, "first": "none", "second": "centred", "gate": "row", "act": "none", "stream": True, "type": "f32", "pad": 0},
        # The gradient of a training batch, gates of their own for every entry.
        {"name": "norm_grad_train", "op": "norm_grad", "n": 8192, "m": 4096, "first": "rms", "second": "rms", "gate": "rows", "act": "silu", "stream": True, "type": "bf16", "pad": 0},
        # A few rows of a served model: most groups have one row or none, the weights' bytes count.
        {"name": "grouped_serve", "op": "grouped", "groups": 16, "n": 8, "k": 2048, "m": 2048, "act": "silu", "keep": False, "keys": "u", "tail": 0, "type": "bf16", "pad": 0},
        # 10,000 joined rows of 220 columns with a layer of 256 for each of 64 keys, skewed, padded with rows of no group.
        {"name": "grouped_join", "op": "grouped", "groups": 64, "n": 10_000, "k": 220, "m": 256, "act": "relu", "keep": True, "keys": "z", "tail": 100, "type": "f32", "pad": 0},
        # The wide layers of a training batch, eight groups of skewed sizes.
        {"name": "grouped_train", "op": "grouped", "groups": 8, "n": 16_384, "k": 2048, "m": 4096, "act": "gelu", "keep": True, "keys": "z", "tail": 0, "type": "bf16", "pad": 0},
        # Small odd layers for 40 keys: the gradient of a mini-batch.
        {"name": "grouped_grad_ragged", "op": "grouped_grad", "groups": 40, "n": 5003, "k": 333, "m": 129, "act": "sigmoid", "keys": "z", "tail": 0, "type": "f32", "pad": 0},
        # The gradient of the wide layers.
        {"name": "grouped_grad_train", "op": "grouped_grad", "groups": 8, "n": 16_384, "k": 2048, "m": 4096, "act": "gelu", "keys": "z", "tail": 0, "type": "bf16", "pad": 0},
        # The gradients of a small model: latency.
        {"name": "clip_small", "op": "clip", "count": 12, "width": 64, "clip": 0.5, "type": "f32", "pad": 0},
        # The gradients of a large one, 630 MB.
        {"name": "clip_large", "op": "clip", "count": 60, "width": 2048, "clip": 0.5, "type": "bf16", "pad": 0},
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 64:
        v -= v % 32                      # half of the sizes are the round ones that programs choose
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "grouped", "grouped_grad", "clip"])
    c = {"op": op, "type": rng.choice(["f32", "bf16"]), "pad": rng.choice([0, 0, 0, 1, 8])}
    if op in ("norm", "norm_grad"):
        c["m"] = _log(rng, 8, 8192)
        most = 30_000_000 if c["type"] == "bf16" else 15_000_000
        c["n"] = _log(rng, 1, max(1, min(200_000, most // c["m"])))
        c.update(first=rng.choice(["none", "rms", "centred"]), second=rng.choice(["none", "rms", "centred"]), gate=rng.choice(["none", "row", "rows"]),
                 act=rng.choice(["none", "sigmoid", "silu"]), stream=rng.random() < 0.8)
        if c["first"] == "none" and c["second"] == "none":
            c["first"] = "rms"
    elif op in ("grouped", "grouped_grad"):
        # one row to large batches; products of at most the largest listed ones in bfloat16, a fifth of them in float32
        top = 2.7e11 if c["type"] == "bf16" else 5e10
        c.update(groups=_log(rng, 1, 128), n=_log(rng, 1, 16_384), k=_log(rng, 16, 4096), act=rng.choice(["none", "relu", "sigmoid", "silu", "gelu"]))
        most = min(top / (2 * c["n"] * c["k"]), 64e6 / (c["groups"] * c["k"]))
        c["m"] = _log(rng, 16, max(16, min(4096, int(most))))
        c.update(keys=rng.choice("uz"), tail=rng.choice([0, 0, min(c["n"] // 3, 17)]))
        if op == "grouped":
            c["keep"] = rng.random() < 0.5
    else:
        c.update(width=_log(rng, 16, 2048), clip=rng.choice([0.1, 0.5, 2.0, 0.0]))
        c["count"] = _log(rng, 1, max(1, min(60, int(250e6 / (1.3 * c["width"] ** 2)))))
    return c


# ------------------------------------------------------------------------------------------------------------ inputs
def _randn(shape, gen, scale=1.0):
    return torch.randn(shape, generator=gen, device=DEV) * scale


def _matrix(x, dtype, pad):
    """x as the caller holds it: in its type, a column slice of a wider matrix where pad > 0."""
    if pad == 0:
        return x.to(dtype)
    wide = torch.zeros(*x.shape[:-1], x.shape[-1] + pad, dtype=dtype, device=DEV)
    wide[..., : x.shape[-1]] = x.to(dtype)
    return wide[..., : x.shape[-1]]


def _shares(case):
    """The probability of each group."""
    w = torch.arange(1, case["groups"] + 1, dtype=torch.float64).pow(-1.1 if case["keys"] == "z" else 0.0)
    return w / w.sum()


def _offsets(case, gen):
    """Where the rows of each group begin, with the end of the last: rows sorted by a key that is drawn for each."""
    cdf = torch.cumsum(_shares(case), 0).to(DEV)
    u = torch.rand(case["n"] - case["tail"], generator=gen, device=DEV, dtype=torch.float64)
    ids = torch.searchsorted(cdf, u).clamp(max=case["groups"] - 1)
    ids = torch.randperm(case["groups"], generator=gen, device=DEV)[ids]
    sizes = torch.bincount(ids, minlength=case["groups"])
    return torch.cat([torch.zeros(1, dtype=sizes.dtype, device=DEV), torch.cumsum(sizes, 0)]).int()


def _shapes(case):
    """The tensors of a model of this width: square and wide matrices, vectors and small odd matrices."""
    d = case["width"]
    return [((d, d), (d,), (d, 4 * d), (d // 3 + 1, 7))[i % 4] for i in range(case["count"])]


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    op, dt, pad = case["op"], DTYPES[case["type"]], case["pad"]
    s = {"case": dict(case)}
    if op in ("norm", "norm_grad"):
        n, m = case["n"], case["m"]
        s["h"] = _matrix(_randn((n, m), gen, 2.0) + 0.5, dt, pad)
        s["x"] = _matrix(_randn((n, m), gen, 3.0), dt, pad) if case["stream"] else None
        s["gate"] = {"none": None, "row": lambda: _randn((m,), gen, 0.5).to(dt), "rows": lambda: _matrix(_randn((n, m), gen), dt, pad)}[case["gate"]]
        s["gate"] = s["gate"]() if s["gate"] is not None else None
        for which in ("first", "second"):
            s["gain_" + which] = (1.0 + _randn((m,), gen, 0.2)).to(dt) if case[which] != "none" else None
            s["bias_" + which] = _randn((m,), gen, 0.1).to(dt) if case[which] == "centred" else None
        s["scale"] = 0.7
        if op == "norm_grad":
            s["d_r"] = _matrix(_randn((n, m), gen, GRAD), dt, pad)
            s["d_y"] = _matrix(_randn((n, m), gen, GRAD), dt, pad) if case["second"] != "none" else None
    elif op in ("grouped", "grouped_grad"):
        g, n, k, m = case["groups"], case["n"], case["k"], case["m"]
        s["offsets"] = _offsets(case, gen)
        s["X"] = _matrix(_randn((n, k), gen), dt, pad)
        s["W"] = _matrix(_randn((g, k, m), gen, 1.0 / math.sqrt(k)), dt, pad)
        if op == "grouped":
            s["bias"] = _randn((g, m), gen, 0.1).to(dt)
        else:
            s["pre"] = _matrix(_randn((n, m), gen), dt, pad) if case["act"] != "none" else None
            s["d_out"] = _matrix(_randn((n, m), gen, 1e-2), dt, pad)
    else:
        s["tensors"] = []
        for shape in _shapes(case):
            t = _randn(shape, gen, GRAD)
            s["tensors"].append(t if len(shape) == 1 else _matrix(t, dt, pad))
        total = sum(t.numel() for t in s["tensors"])
        # half of the norm that such gradients have, twice of it, or no limit at all
        s["max_norm"] = case["clip"] * GRAD * math.sqrt(total) if case["clip"] > 0 else math.inf
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op, dt = case["op"], DTYPES[case["type"]]
    new = lambda *shape: torch.empty(*shape, dtype=dt, device=DEV)
    # the buffers that a training or serving loop keeps from step to step
    if op == "norm":
        s["r"] = new(case["n"], case["m"])
        s["y"] = new(case["n"], case["m"]) if case["second"] != "none" else None
    elif op == "norm_grad":
        for key in ("h", "x", "gate", "gain_first", "bias_first", "gain_second", "bias_second"):
            s["d_" + key] = new(*s[key].shape) if s[key] is not None else None
    elif op in ("grouped", "grouped_grad"):
        g, n, k, m = case["groups"], case["n"], case["k"], case["m"]
        # rows of no group stay as they are, here zeros
        if op == "grouped":
            s["out"] = new(n, m).zero_()
            s["pre"] = new(n, m).zero_() if case["keep"] else None
        else:
            s["d_X"], s["d_W"], s["d_bias"] = new(n, k).zero_(), new(g, k, m), new(g, m)
        s["starts"] = s["offsets"].tolist()              # for the loop over the groups of the plain form
    else:
        s["outs"] = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in s["tensors"]] if case["clip"] > 0 else None
        s["norm"] = torch.empty(1, device=DEV)
    if own:
        import paper_2502_01985_amd as il
        if op == "clip":
            s["list"] = il.TensorList(s["tensors"], s["outs"])
        s["workspace"] = torch.empty(_workspace_bytes(il, s), dtype=torch.uint8, device=DEV)
    return s


def _workspace_bytes(il, s):
    c = s["case"]
    op = c["op"]
    if op == "norm":
        return 0
    if op == "norm_grad":
        return il.ilargi_norm_grad_workspace_bytes(c["n"], c["m"], DTYPES[c["type"]])
    if op == "clip":
        return il.ilargi_clip_norm_workspace_bytes(s["list"])
    forward, gradient = il.ilargi_grouped_linear_workspace_bytes(c["groups"], c["n"], c["k"], c["m"], DTYPES[c["type"]])
    return forward if op == "grouped" else gradient


# ----------------------------------------------------------------------------------------------------------- one pass
NORM_GRADS = ("d_h", "d_x", "d_gate", "d_gain_first", "d_bias_first", "d_gain_second", "d_bias_second")


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2502_01985_amd as il
    c = s["case"]
    op = c["op"]
    if op in ("norm", "norm_grad"):
        block = dict(first=c["first"], gain1=s["gain_first"], bias1=s["bias_first"], gate=s["gate"], gate_act=c["act"], scale=s["scale"], x=s["x"],
                     second=c["second"], gain2=s["gain_second"], bias2=s["bias_second"], eps=EPS)
        if op == "norm":
            r, y = il.ilargi_norm(s["h"], r=s["r"], y=s["y"], **block)
            return {"r": r, "y": y}
        got = il.ilargi_norm_grad(s["d_r"], s["d_y"], s["h"], d_h=s["d_h"], d_x=s["d_x"], d_gate=s["d_gate"], d_gain1=s["d_gain_first"],
                                  d_bias1=s["d_bias_first"], d_gain2=s["d_gain_second"], d_bias2=s["d_bias_second"], workspace=s["workspace"], **block)
        return dict(zip(NORM_GRADS, got))
    if op == "grouped":
        out = il.ilargi_grouped_linear(s["X"], s["W"], s["offsets"], bias=s["bias"], act=c["act"], out=s["out"], pre=s["pre"], workspace=s["workspace"])
        return {"out": out, "pre": s["pre"]}
    if op == "grouped_grad":
        d_X, d_W, d_bias = il.ilargi_grouped_linear_grad(s["d_out"], s["X"], s["W"], s["offsets"], pre=s["pre"], act=c["act"], d_X=s["d_X"],
                                                         d_W=s["d_W"], d_bias=s["d_bias"], workspace=s["workspace"])
        return {"d_X": d_X, "d_W": d_W, "d_bias": d_bias}
    norm = il.ilargi_clip_norm(s["list"], s["max_norm"], norm=s["norm"], workspace=s["workspace"])
    return [norm, *(s["outs"] or [])]


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "sigmoid":
        e = 1.0 / (1.0 + torch.exp(-z))
        return e * (1.0 - e)
    if act == "silu":
        e = 1.0 / (1.0 + torch.exp(-z))
        return e * (1.0 + z * (1.0 - e))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _unit(v, kind):
    """v normalised, before gain and bias, and what it was divided by, reversed."""
    if kind == "none":
        return v, None
    if kind == "centred":
        v = v - v.sum(1, keepdim=True) / v.shape[1]
    by = 1.0 / torch.sqrt((v * v).sum(1, keepdim=True) / v.shape[1] + EPS)
    return v * by, by


def _affine(v, gain, bias):
    if gain is not None:
        v = v * gain.float()
    return v + bias.float() if bias is not None else v


def _unit_grad(t, unit, by, kind):
    if kind == "none":
        return t
    m = t.shape[1]
    back = t - unit * ((t * unit).sum(1, keepdim=True) / m)
    if kind == "centred":
        back = back - t.sum(1, keepdim=True) / m
    return back * by


def _run_plain(s):
    c = s["case"]
    op, dt = c["op"], DTYPES[c["type"]]
    if op in ("norm", "norm_grad"):
        unit1, by1 = _unit(s["h"].float(), c["first"])
        u = _affine(unit1, s["gain_first"], s["bias_first"])
        gate = s["gate"].float() if s["gate"] is not None else None
        r = s["scale"] * (u if gate is None else _act(gate, c["act"]) * u)
        if s["x"] is not None:
            r = r + s["x"].float()
        unit2, by2 = _unit(r, c["second"])
        if op == "norm":
            return {"r": r.to(dt), "y": _affine(unit2, s["gain_second"], s["bias_second"]).to(dt) if c["second"] != "none" else None}
        out = dict.fromkeys(NORM_GRADS)
        dr = s["d_r"].float()
        if s["d_y"] is not None:
            dy = s["d_y"].float()
            out["d_gain_second"] = (dy * unit2).sum(0).to(dt)
            if s["bias_second"] is not None:
                out["d_bias_second"] = dy.sum(0).to(dt)
            dr = dr + _unit_grad(dy * s["gain_second"].float(), unit2, by2, c["second"])
        if s["x"] is not None:
            out["d_x"] = dr.to(dt)
        du = s["scale"] * dr
        if gate is not None:
            d_gate = du * u * _act_grad(gate, c["act"])
            out["d_gate"] = (d_gate.sum(0) if c["gate"] == "row" else d_gate).to(dt)
            du = du * _act(gate, c["act"])
        if s["gain_first"] is not None:
            out["d_gain_first"] = (du * unit1).sum(0).to(dt)
        if s["bias_first"] is not None:
            out["d_bias_first"] = du.sum(0).to(dt)
        t = du * s["gain_first"].float() if s["gain_first"] is not None else du
        out["d_h"] = _unit_grad(t, unit1, by1, c["first"]).to(dt)
        return out
    if op in ("grouped", "grouped_grad"):
        g, n, k, m, at = c["groups"], c["n"], c["k"], c["m"], s["starts"]
        if op == "grouped":
            z = torch.zeros(n, m, device=DEV)
            for j in range(g):
                if at[j + 1] > at[j]:
                    z[at[j]: at[j + 1]] = s["X"][at[j]: at[j + 1]].float() @ s["W"][j].float() + s["bias"][j].float()
            out = _act(z, c["act"])
            out[at[g]:] = 0.0
            return {"out": out.to(dt), "pre": z.to(dt) if c["keep"] else None}
        grad = s["d_out"].float()
        if s["pre"] is not None:
            grad = grad * _act_grad(s["pre"].float(), c["act"])
        d_X, d_W, d_bias = torch.zeros(n, k, device=DEV), torch.zeros(g, k, m, device=DEV), torch.zeros(g, m, device=DEV)
        for j in range(g):
            rows = slice(at[j], at[j + 1])
            if at[j + 1] > at[j]:
                d_X[rows] = grad[rows] @ s["W"][j].float().t()
                d_W[j] = s["X"][rows].float().t() @ grad[rows]
                d_bias[j] = grad[rows].sum(0)
        return {"d_X": d_X.to(dt), "d_W": d_W.to(dt), "d_bias": d_bias.to(dt)}
    total = torch.zeros((), dtype=torch.float64, device=DEV)
    for t in s["tensors"]:
        total = total + (t.float() * t.float()).sum(dtype=torch.float64)      # (float32 sums of so many squares lose what matters)
    norm = torch.sqrt(total).float().reshape(1)
    if s["outs"] is None:
        return [norm]
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    return [norm, *((t.float() * factor).to(t.dtype) for t in s["tensors"])]


# ------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    d64 = lambda t: t.double() if t is not None else None
    if op in ("norm", "norm_grad"):
        h, x, gate, g1, b1, g2, b2 = (d64(s[k]) for k in ("h", "x", "gate", "gain_first", "bias_first", "gain_second", "bias_second"))
        st1 = _stats(h, case["first"])
        a, a_slope = _smooth(gate, case["act"]) if gate is not None else (torch.ones(1, case["m"], dtype=torch.float64, device=DEV), None)
        u = _scaled(h, st1, g1, b1)
        r = torch.addcmul(x if x is not None else torch.zeros_like(h), u, a, value=s["scale"])
        st2 = _stats(r, case["second"])
        if op == "norm":
            return {"r": r, "y": _scaled(r, st2, g2, b2) if case["second"] != "none" else None}
        out = dict.fromkeys(NORM_GRADS)
        dr = s["d_r"].double()
        if s["d_y"] is not None:
            dy = s["d_y"].double()
            out["d_gain_second"] = torch.einsum("ij,ij->j", dy, _scaled(r, st2, None, None))
            if b2 is not None:
                out["d_bias_second"] = dy.sum(0)
            dr = dr + _back(dy * g2, r, st2)
        if x is not None:
            out["d_x"] = dr
        if gate is not None:
            per = s["scale"] * dr * u * a_slope
            out["d_gate"] = per.sum(0) if case["gate"] == "row" else per
        du = dr * a * s["scale"]
        if g1 is not None:
            out["d_gain_first"] = torch.einsum("ij,ij->j", du, _scaled(h, st1, None, None))
            du = du * g1
        if b1 is not None:
            out["d_bias_first"] = (dr * a * s["scale"]).sum(0)
        out["d_h"] = _back(du, h, st1)
        return out
    if op in ("grouped", "grouped_grad"):
        g, n, k, m = case["groups"], case["n"], case["k"], case["m"]
        at = s["offsets"].tolist()
        parts = [slice(a, b) for a, b in zip(at[:-1], at[1:])]
        X = s["X"].double()
        if op == "grouped":
            z = torch.zeros(n, m, dtype=torch.float64, device=DEV)
            out = torch.zeros_like(z)
            for j, p in enumerate(parts):
                z[p] = torch.addmm(s["bias"][j].double(), X[p], s["W"][j].double())
                out[p] = _smooth(z[p], case["act"])[0]
            return {"out": out, "pre": z if case["keep"] else None}
        d = s["d_out"].double()
        if s["pre"] is not None:
            d = d * _smooth(s["pre"].double(), case["act"])[1]
        d_X = torch.zeros(n, k, dtype=torch.float64, device=DEV)
        d_W = torch.zeros(g, k, m, dtype=torch.float64, device=DEV)
        d_bias = torch.zeros(g, m, dtype=torch.float64, device=DEV)
        for j, p in enumerate(parts):
            if p.stop > p.start:
                d_X[p] = d[p] @ s["W"][j].double().t().contiguous()
                d_W[j] = X[p].t().contiguous() @ d[p]
                d_bias[j] = d[p].sum(0)
        return {"d_X": d_X, "d_W": d_W, "d_bias": d_bias}
    norm = torch.stack([torch.linalg.vector_norm(t.double()) for t in s["tensors"]]).square().sum().sqrt()
    if case["clip"] <= 0:
        return [norm.reshape(1)]
    factor = (s["max_norm"] / norm).clamp(max=1.0)
    return [norm.reshape(1), *(t.double() * factor for t in s["tensors"])]


def _stats(v, kind):
    """The mean that is subtracted and the deviation that is divided by, a column each."""
    if kind == "none":
        return None
    var, mean = (v.square().mean(1, keepdim=True), torch.zeros(v.shape[0], 1, dtype=v.dtype, device=v.device))
    if kind == "centred":
        mean = v.mean(1, keepdim=True)
        var = (v - mean).square().mean(1, keepdim=True)
    return mean, (var + EPS).sqrt(), kind == "centred"


def _scaled(v, stats, gain, bias):
    if stats is not None:
        v = (v - stats[0]) / stats[1]
    if gain is not None:
        v = v * gain
    return v + bias if bias is not None else v


def _back(t, v, stats):
    if stats is None:
        return t
    mean, dev, centred = stats
    c = v - mean
    out = (t - c * (t * c).mean(1, keepdim=True) / dev.square()) / dev
    return out - t.mean(1, keepdim=True) / dev if centred else out


def _smooth(z, act):
    """f(z) and f'(z)."""
    if act == "relu":
        return z.clamp(min=0), torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
    if act in ("sigmoid", "silu"):
        p = torch.special.expit(z)
        return (p, p * torch.special.expit(-z)) if act == "sigmoid" else (z * p, p + z * p * torch.special.expit(-z))
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


# --------------------------------------------------------------------------------------------------------------- work
def work(case):
    op, b = case["op"], BYTES[case["type"]]
    if op in ("norm", "norm_grad"):
        n, m = case["n"], case["m"]
        vectors = sum({"none": 0, "rms": 1, "centred": 2}[case[w]] for w in ("first", "second")) + (case["gate"] == "row")
        second, rows = case["second"] != "none", case["gate"] == "rows"
        if op == "norm":
            return {"bytes": b * (n * m * (2 + case["stream"] + rows + second) + vectors * m), "flops": 12 * n * m}
        # h, the stream and the gate are read with the gradients of r and y; those of h, the stream and the gate are written
        return {"bytes": b * (n * m * (3 + 2 * case["stream"] + 2 * rows + second) + 2 * vectors * m), "flops": 30 * n * m}
    if op in ("grouped", "grouped_grad"):
        g, k, m, n = case["groups"], case["k"], case["m"], case["n"] - case["tail"]
        used = float((1.0 - (1.0 - _shares(case)).pow(n)).sum())         # groups that have rows, on average
        if op == "grouped":
            return {"bytes": int(b * (n * k + used * k * m + used * m + n * m * (1 + case["keep"])) + 4 * g), "flops": 2 * n * k * m}
        return {"bytes": int(b * (2 * n * k + (used + g) * k * m + g * m + n * m * (1 + (case["act"] != "none"))) + 4 * g), "flops": 4 * n * k * m}
    count = lambda shape: math.prod(shape)
    read = sum(count(t) * (4 if len(t) == 1 else b) for t in _shapes(case))
    return {"bytes": read * (2 if case["clip"] > 0 else 1) + 4, "flops": 3 * sum(count(t) for t in _shapes(case))}
