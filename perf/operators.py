"""The operators of a model with learned features over a join, as measurable cases.

  embed        rows of a learned table picked by foreign keys, scaled
  embed_grad   the gradient of that table: rows of the output's gradient summed by key
  linear       f(X W + bias) + residual, with the values before f where training keeps them
  linear_grad  the gradients of X, W and the bias
  orthogonalize  an update matrix brought near its orthogonal factor by Newton-Schulz products

`run` computes each of them with elementary torch operations in 32 bits (`own` false) or through this package's entry
points (`own` true).  `exact` is the definition in 64 bits.

Every case has the element `type` ("f32" or "bf16") and `pad`, the columns that the caller's matrices have beyond the ones
used (the operands are then column slices of wider tensors).  `keys` is "u" (uniform) or "z" (Zipf 1.1); `missing` the
share of the rows whose key finds no row (-1).
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
COEF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def listed():
    return [
        # Scoring one small batch of joined rows: 512 keys into a table as long as the smallest joined one.
        {"name": "embed_small", "op": "embed", "n": 512, "rows": 1000, "cols": 64, "type": "f32", "keys": "u", "missing": 0.0, "pad": 0},
        # Every row of a join of a million rows takes its learned row: skewed keys, a table of 100,000 rows.
        {"name": "embed_join", "op": "embed", "n": 1_000_000, "rows": 100_000, "cols": 256, "type": "bf16", "keys": "z", "missing": 0.0, "pad": 0},
        # A mini-batch against the shorter one-hot table of the benchmark, odd row length, one key in ten unmatched.
        {"name": "embed_grad_ragged", "op": "embed_grad", "n": 9001, "rows": 6040, "cols": 75, "type": "f32", "keys": "z", "missing": 0.1, "pad": 0},
        # The gradient over the whole join: a million rows, skewed keys.
        {"name": "embed_grad_join", "op": "embed_grad", "n": 1_000_000, "rows": 100_000, "cols": 128, "type": "bf16", "keys": "z", "missing": 0.0, "pad": 0},
        # One row through a layer: serving, where the weights' bytes and the launch count.
        {"name": "linear_one_row", "op": "linear", "n": 1, "k": 4096, "m": 4096, "act": "silu", "residual": True, "keep": False, "type": "bf16", "pad": 0},
        # A few rows with odd lengths in float32: the joined columns of one schema, unaligned.
        {"name": "linear_ragged", "op": "linear", "n": 1003, "k": 333, "m": 517, "act": "relu", "residual": False, "keep": True, "type": "f32", "pad": 0},
        # The wide layer of a training step, values before the activation kept for the gradient.
        {"name": "linear_train", "op": "linear", "n": 16384, "k": 2048, "m": 8192, "act": "gelu", "residual": False, "keep": True, "type": "bf16", "pad": 0},
        # A hidden layer on 220 joined columns for 10,000 rows, float32.
        {"name": "linear_grad_join", "op": "linear_grad", "n": 10_000, "k": 220, "m": 256, "act": "sigmoid", "type": "f32", "pad": 0},
        # The gradient of a wide square layer.
        {"name": "linear_grad_train", "op": "linear_grad", "n": 8192, "k": 4096, "m": 4096, "act": "gelu", "type": "bf16", "pad": 0},
        # The updates of four small layers at once: latency.
        {"name": "ortho_small", "op": "orthogonalize", "batch": 4, "rows": 220, "cols": 64, "steps": 5, "type": "f32", "pad": 0},
        # One layer's update, four times as wide as tall, gradients in bfloat16.
        {"name": "ortho_wide", "op": "orthogonalize", "batch": 1, "rows": 1024, "cols": 4096, "steps": 5, "type": "bf16", "pad": 0},
        # The update of a large square layer in float32.
        {"name": "ortho_square", "op": "orthogonalize", "batch": 1, "rows": 2048, "cols": 2048, "steps": 5, "type": "f32", "pad": 0},
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 64:
        v -= v % 32                      # half of the sizes are the round ones that programs choose
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "linear", "linear_grad", "orthogonalize"])
    c = {"op": op, "type": rng.choice(["f32", "bf16"]), "pad": rng.choice([0, 0, 0, 1, 8])}
    if op in ("embed", "embed_grad"):
        c.update(rows=_log(rng, 100, 200_000), cols=_log(rng, 8, 1024), keys=rng.choice("uz"), missing=rng.choice([0.0, 0.0, 0.1]))
        c["n"] = _log(rng, 64, max(64, min(1_000_000, 100_000_000 // c["cols"])))
    elif op in ("linear", "linear_grad"):
        # one row to large batches; products of at most a fifth of the largest listed ones in float32
        top = 5e11 if c["type"] == "bf16" else 1e11
        c.update(n=_log(rng, 1, 16384), k=_log(rng, 16, 8192), act=rng.choice(["none", "relu", "sigmoid", "silu", "gelu"]))
        most = top / (2 * c["n"] * c["k"]) / (2 if op == "linear_grad" else 1)
        c["m"] = _log(rng, 16, max(16, min(8192, int(most))))
        if op == "linear":
            c.update(residual=rng.random() < 0.5, keep=rng.random() < 0.5)
    else:
        c.update(rows=_log(rng, 16, 2048), cols=_log(rng, 16, 2048), steps=5)
        c["batch"] = rng.randint(1, max(1, min(8, int(2048 * 2048 // (c["rows"] * c["cols"])))))
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


def _keys(case, gen):
    n, rows = case["n"], case["rows"]
    u = torch.rand(n, generator=gen, device=DEV, dtype=torch.float64)
    if case["keys"] == "z":
        cdf = torch.cumsum(torch.arange(1, rows + 1, device=DEV, dtype=torch.float64).pow(-1.1), 0)
        rank = torch.searchsorted(cdf / cdf[-1], u).clamp(max=rows - 1)
        ids = torch.randperm(rows, generator=gen, device=DEV)[rank]
    else:
        ids = (u * rows).long().clamp(max=rows - 1)
    if case["missing"] > 0:
        ids[torch.rand(n, generator=gen, device=DEV) < case["missing"]] = -1
    return ids.int()


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    op, dt, pad = case["op"], DTYPES[case["type"]], case["pad"]
    s = {"case": dict(case)}
    if op == "embed":
        s["ids"] = _keys(case, gen)
        s["table"] = _matrix(_randn((case["rows"], case["cols"]), gen, 0.02), dt, pad)
        s["scale"] = math.sqrt(case["cols"])
    elif op == "embed_grad":
        s["ids"] = _keys(case, gen)
        s["d_out"] = _matrix(_randn((case["n"], case["cols"]), gen, 1e-3), dt, pad)
        s["scale"] = math.sqrt(case["cols"])
    elif op in ("linear", "linear_grad"):
        n, k, m = case["n"], case["k"], case["m"]
        s["X"] = _matrix(_randn((n, k), gen), dt, pad)
        s["W"] = _matrix(_randn((k, m), gen, 1.0 / math.sqrt(k)), dt, pad)
        if op == "linear":
            s["bias"] = _randn((m,), gen, 0.1).to(dt)
            s["residual"] = _matrix(_randn((n, m), gen), dt, pad) if case["residual"] else None
        else:
            s["pre"] = _matrix(_randn((n, m), gen), dt, pad) if case["act"] != "none" else None
            s["d_out"] = _matrix(_randn((n, m), gen, 1e-2), dt, pad)
    else:
        # gradients of layers: a few strong directions over noise
        p, q, b = case["rows"], case["cols"], case["batch"]
        r = max(1, min(p, q) // 8)
        u, v = _randn((b, p, r), gen), _randn((b, r, q), gen)
        s["G"] = _matrix((torch.bmm(u, v) / math.sqrt(r) + 0.3 * _randn((b, p, q), gen)) * 1e-3, dt, pad)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op, dt = case["op"], DTYPES[case["type"]]
    # the buffers that a training or serving loop keeps from step to step
    if op == "embed":
        s["out"] = torch.empty(case["n"], case["cols"], dtype=dt, device=DEV)
    elif op == "embed_grad":
        s["d_table"] = torch.empty(case["rows"], case["cols"], dtype=dt, device=DEV)
    elif op == "linear":
        s["out"] = torch.empty(case["n"], case["m"], dtype=dt, device=DEV)
        s["pre"] = torch.empty(case["n"], case["m"], dtype=dt, device=DEV) if case["keep"] else None
    elif op == "linear_grad":
        s["d_X"] = torch.empty(case["n"], case["k"], dtype=dt, device=DEV)
        s["d_W"] = torch.empty(case["k"], case["m"], dtype=dt, device=DEV)
        s["d_bias"] = torch.empty(case["m"], dtype=dt, device=DEV)
    else:
        s["out"] = torch.empty(case["batch"], case["rows"], case["cols"], dtype=dt, device=DEV)
    if own:
        import paper_2502_01985_amd as il
        s["workspace"] = torch.empty(_workspace_bytes(il, case), dtype=torch.uint8, device=DEV)
    return s


def _workspace_bytes(il, case):
    op = case["op"]
    if op == "embed":
        return 0
    if op == "embed_grad":
        return il.ilargi_embed_grad_workspace_bytes(case["n"], case["rows"], case["cols"])
    if op in ("linear", "linear_grad"):
        forward, gradient = il.ilargi_linear_workspace_bytes(case["n"], case["k"], case["m"], DTYPES[case["type"]])
        return forward if op == "linear" else gradient
    return il.ilargi_orthogonalize_workspace_bytes(case["batch"], case["rows"], case["cols"], DTYPES[case["type"]])


# ----------------------------------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2502_01985_amd as il
    c = s["case"]
    op = c["op"]
    if op == "embed":
        return il.ilargi_embed(s["table"], s["ids"], scale=s["scale"], out=s["out"])
    if op == "embed_grad":
        return il.ilargi_embed_grad(s["d_out"], s["ids"], c["rows"], scale=s["scale"], d_table=s["d_table"], workspace=s["workspace"])
    if op == "linear":
        out = il.ilargi_linear(s["X"], s["W"], bias=s["bias"], residual=s["residual"], act=c["act"], out=s["out"], pre=s["pre"],
                               workspace=s["workspace"])
        return {"out": out, "pre": s["pre"]}
    if op == "linear_grad":
        d_X, d_W, d_bias = il.ilargi_linear_grad(s["d_out"], s["X"], s["W"], pre=s["pre"], act=c["act"], d_X=s["d_X"], d_W=s["d_W"],
                                                 d_bias=s["d_bias"], workspace=s["workspace"])
        return {"d_X": d_X, "d_W": d_W, "d_bias": d_bias}
    return il.ilargi_orthogonalize(s["G"], steps=c["steps"], coef=COEF, eps=EPS, out=s["out"], workspace=s["workspace"])


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
    return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))


def _run_plain(s):
    c = s["case"]
    op, dt = c["op"], DTYPES[c["type"]]
    if op == "embed":
        ids = s["ids"]
        rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
        return torch.where((ids >= 0)[:, None], rows, 0.0).to(dt)
    if op == "embed_grad":
        ids = s["ids"]
        g = torch.where((ids >= 0)[:, None], s["d_out"].float() * s["scale"], 0.0)
        return torch.zeros(c["rows"], c["cols"], device=DEV).index_add_(0, ids.clamp(min=0), g).to(dt)
    if op == "linear":
        z = s["X"].float() @ s["W"].float() + s["bias"].float()
        out = _act(z, c["act"])
        if s["residual"] is not None:
            out = out + s["residual"].float()
        return {"out": out.to(dt), "pre": z.to(dt) if c["keep"] else None}
    if op == "linear_grad":
        g = s["d_out"].float()
        if c["act"] != "none":
            g = g * _act_grad(s["pre"].float(), c["act"])
        return {"d_X": (g @ s["W"].float().t()).to(dt), "d_W": (s["X"].float().t() @ g).to(dt), "d_bias": g.sum(0).to(dt)}
    return _orthogonal(s["G"].float(), c["steps"]).to(dt)


def _orthogonal(X, steps):
    tall = X.shape[1] > X.shape[2]
    if tall:
        X = X.transpose(1, 2)
    a, b, c = COEF
    X = (X / (X.square().sum((1, 2), keepdim=True).sqrt() + EPS)).contiguous()
    for _ in range(steps):
        A = torch.bmm(X, X.transpose(1, 2).contiguous())
        X = a * X + torch.bmm(b * A + c * torch.bmm(A, A), X)
    return X.transpose(1, 2) if tall else X


# ------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "embed":
        t = torch.cat([s["table"].double(), torch.zeros(1, case["cols"], dtype=torch.float64, device=DEV)])
        return t[s["ids"].long()] * s["scale"]           # -1 picks the last, empty row
    if op == "embed_grad":
        out = torch.zeros(case["rows"] + 1, case["cols"], dtype=torch.float64, device=DEV)
        ids = torch.where(s["ids"] < 0, case["rows"], s["ids"]).long()
        out.index_put_((ids,), s["d_out"].double(), accumulate=True)
        return out[:-1] * s["scale"]
    if op == "linear":
        z = torch.addmm(s["bias"].double(), s["X"].double(), s["W"].double())
        out = _smooth(z, case["act"])[0]
        if s["residual"] is not None:
            out = out + s["residual"].double()
        return {"out": out, "pre": z if case["keep"] else None}
    if op == "linear_grad":
        g = s["d_out"].double()
        if s["pre"] is not None:
            g = g * _smooth(s["pre"].double(), case["act"])[1]
        one = torch.ones(1, case["n"], dtype=torch.float64, device=DEV)
        return {"d_X": g @ s["W"].double().t().contiguous(), "d_W": s["X"].double().t().contiguous() @ g, "d_bias": (one @ g)[0]}
    G = s["G"].double()
    a, b, c = COEF
    out = []
    for g in G:                                           # matrix by matrix, the shorter side in front
        t = g.t().contiguous() if g.shape[0] > g.shape[1] else g
        t = t / (torch.linalg.norm(t) + EPS)
        for _ in range(case["steps"]):
            A = t @ t.t().contiguous()
            t = a * t + b * (A @ t) + c * (A @ (A @ t))
        out.append(t.t() if g.shape[0] > g.shape[1] else t)
    return torch.stack(out)


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
    if op == "embed":
        n, d = case["n"], case["cols"]
        return {"bytes": 4 * n + min(n, case["rows"]) * d * b + n * d * b, "flops": n * d}
    if op == "embed_grad":
        n, d = case["n"], case["cols"]
        return {"bytes": 4 * n + n * d * b + case["rows"] * d * b, "flops": n * d}
    if op in ("linear", "linear_grad"):
        n, k, m = case["n"], case["k"], case["m"]
        if op == "linear":
            return {"bytes": b * (n * k + k * m + m + n * m * (1 + case["residual"] + case["keep"])), "flops": 2 * n * k * m}
        return {"bytes": b * (2 * n * k + 2 * k * m + m + n * m * (1 + (case["act"] != "none"))), "flops": 4 * n * k * m}
    s, l = sorted((case["rows"], case["cols"]))
    # the two symmetric products of a step are formed once for both triangles
    return {"bytes": 2 * case["batch"] * s * l * b, "flops": case["batch"] * case["steps"] * (3 * s * s * l + s * s * s)}
