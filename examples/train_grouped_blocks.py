"""Trains a deeper model on a star join that is never built: a block of layers of its own for every row of a small joined table.

    H = T W0                                      one row for each row of the join, in the order of its key from here on
    A = silu(N(H) W1[key] + b1[key]),  O = A W2[key]
    R = H + g o N(O),   p = sigmoid(N(R) w + b)   N: v / sqrt(mean v^2 + eps) times a learned gain

T = [S | Q[key]] is a two-table star join (``datagen.star_schema``) whose joined table has few rows (regions, shops, machines).  Its
inverse index (``ilargi_plan_inverse_index``) says which rows of the join belong to which: ``perm`` brings them together
(``ilargi_embed``) and ``rowptr`` is where each group begins (``ilargi_grouped_linear``).  ``ilargi_norm`` normalises the block's output,
adds it to the stream through the gate ``g`` and normalises the sum in one pass.  All gradients are clipped together
(``ilargi_clip_norm``) before plain gradient descent.

    python examples/train_grouped_blocks.py [--rows 100000] [--width 64] [--keys 24] [--steps 30]
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np  # noqa: E402
import torch  # noqa: E402

import datagen  # noqa: E402
import paper_2502_01985_amd as il  # noqa: E402


class GroupedBlockModel:
    """The weights, the gradients, and the buffers that its steps keep."""

    def __init__(self, plan, width, hidden, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
        self.plan, self.n = plan, plan.r_T
        self.starts, self.perm = (torch.from_numpy(v).cuda() for v in il.ilargi_plan_inverse_index(plan, 1))
        keys = self.starts.numel() - 1
        if self.perm.numel() != self.n:
            raise ValueError("every row of the join needs a key")
        ones = lambda m: torch.ones(m, device="cuda")
        self.weights = {"W0": new(plan.c_T, width) / math.sqrt(plan.c_T), "gain1": ones(width), "W1": new(keys, width, hidden) / math.sqrt(width),
                        "b1": torch.zeros(keys, hidden, device="cuda"), "W2": new(keys, hidden, width) / math.sqrt(hidden), "gain2": ones(width),
                        "gate": ones(width) * 0.5, "gain3": ones(width), "w": new(width, 1) / math.sqrt(width), "b": torch.zeros(1, device="cuda")}
        self.grads = {k: torch.empty_like(w) for k, w in self.weights.items()}
        self.clipped = il.TensorList(self.grads.values(), self.grads.values())
        rows = lambda m: torch.empty(self.n, m, device="cuda")
        self.H, self.Hk, self.Y, self.pre, self.A, self.O, self.R, self.Z, self.z, self.p = (rows(m) for m in (width, width, width, hidden, hidden, width, width, width, 1, 1))
        self.norm = torch.empty(1, device="cuda")
        sizes = [*il.ilargi_grouped_linear_workspace_bytes(keys, self.n, width, hidden, torch.float32),
                 *il.ilargi_grouped_linear_workspace_bytes(keys, self.n, hidden, width, torch.float32), il.ilargi_norm_grad_workspace_bytes(self.n, width, torch.float32),
                 *il.ilargi_linear_workspace_bytes(self.n, width, 1, torch.float32), il.ilargi_embed_grad_workspace_bytes(self.n, self.n, width),
                 il.ilargi_clip_norm_workspace_bytes(self.clipped)]
        self.workspace = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")

    def _sum(self):
        """What ``ilargi_norm`` and its gradient are told of the sum R."""
        w = self.weights
        return dict(first="rms", gain1=w["gain2"], gate=w["gate"], x=self.Hk, second="rms", gain2=w["gain3"])

    def forward(self):
        w, ws = self.weights, self.workspace
        il.ilargi_lmm(self.plan, w["W0"], out=self.H)
        il.ilargi_embed(self.H, self.perm, out=self.Hk)
        il.ilargi_norm(self.Hk, first="rms", gain1=w["gain1"], r=self.Y)
        il.ilargi_grouped_linear(self.Y, w["W1"], self.starts, bias=w["b1"], act="silu", out=self.A, pre=self.pre, workspace=ws)
        il.ilargi_grouped_linear(self.A, w["W2"], self.starts, out=self.O, workspace=ws)
        il.ilargi_norm(self.O, r=self.R, y=self.Z, **self._sum())
        il.ilargi_linear(self.Z, w["w"], bias=w["b"], act="sigmoid", out=self.p, pre=self.z, workspace=ws)
        return self.p

    def loss(self, y):
        z = self.z[:, 0].double()
        return float((torch.nn.functional.softplus(z) - y * z).mean())

    def gradients(self, y):
        """Of the mean cross entropy, after ``forward``; ``y`` in the order of the keys.  Into ``grads``."""
        w, g, ws = self.weights, self.grads, self.workspace
        d_z = (self.p - y[:, None]) / self.n
        d_Z, _, _ = il.ilargi_linear_grad(d_z, self.Z, w["w"], d_W=g["w"], d_bias=g["b"], workspace=ws)
        d_O, d_H, *_ = il.ilargi_norm_grad(None, d_Z, self.O, d_gain1=g["gain2"], d_gate=g["gate"], d_gain2=g["gain3"], workspace=ws, **self._sum())
        d_A, _, _ = il.ilargi_grouped_linear_grad(d_O, self.A, w["W2"], self.starts, d_W=g["W2"], d_bias=None, workspace=ws)
        d_Y, _, _ = il.ilargi_grouped_linear_grad(d_A, self.Y, w["W1"], self.starts, pre=self.pre, act="silu", d_W=g["W1"], d_bias=g["b1"], workspace=ws)
        d_N, *_ = il.ilargi_norm_grad(d_Y, None, self.Hk, first="rms", gain1=w["gain1"], d_gain1=g["gain1"], workspace=ws)
        d_H += d_N                                     # the stream's share and the block's
        il.ilargi_tmm(self.plan, il.ilargi_embed_grad(d_H, self.perm, self.n, workspace=ws), out=g["W0"])
        return g

    def step(self, y, lr, max_norm):
        self.forward()
        self.gradients(y)
        il.ilargi_clip_norm(self.clipped, max_norm, norm=self.norm, workspace=self.workspace)
        for k, w in self.weights.items():
            w.sub_(self.grads[k], alpha=lr)


def problem(rows, keys=24, entity_cols=8, joined_cols=4, seed=0):
    """A star join whose labels follow another direction of the entity's columns for every row of the joined table."""
    rng = datagen.rng_for(seed)
    schema = datagen.star_schema(rng, rows, entity_cols, [(keys, joined_cols, ("zipf", 1.1))])
    towards = rng.standard_normal((keys, entity_cols))
    fk = schema.sources[1].row_idx
    logit = (schema.sources[0].D * towards[fk]).sum(1)
    y = (rng.random(rows) < 1.0 / (1.0 + np.exp(-logit))).astype(np.float32)
    return il.schema_to_device(schema), schema, torch.from_numpy(y).cuda()


def train(rows=100_000, width=64, hidden=128, keys=24, steps=30, lr=0.5, max_norm=1.0, seed=0, report=None):
    """Returns the loss before every step and after the last, and the model."""
    sources, schema, y = problem(rows, keys, seed=seed)
    plan = il.ilargi_plan_create(sources, schema.r_T, schema.c_T, max_cx=width)
    model = GroupedBlockModel(plan, width, hidden, seed)
    y = y[model.perm.long()]
    losses = []
    for k in range(steps):
        model.step(y, lr, max_norm)
        losses.append(model.loss(y))
        if report is not None:
            report(k, losses[-1], float(model.norm))
    model.forward()
    losses.append(model.loss(y))
    return losses, model


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rows", type=int, default=100_000)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--keys", type=int, default=24)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    losses, _ = train(a.rows, a.width, keys=a.keys, steps=a.steps, report=lambda k, v, g: print(f"step {k}: loss {v:.4f}, gradient norm {g:.3f}", flush=True))
    print(f"after {a.steps} steps: loss {losses[-1]:.4f}")
