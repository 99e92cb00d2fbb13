"""Trains a small model with learned features on a star join that is never built.

    z = gelu(H W1 + b1) + H,   p = sigmoid(z w2 + b2),   H = T W0 + s E[fk]

T = [S | R[fk]] is a two-table star join (``datagen.star_schema``); E is a learned table with a row for every row of R, picked by
the foreign key.  The products with T run factorized (``ilargi_lmm``, ``ilargi_tmm``), the learned rows and their gradient through
``ilargi_embed`` and ``ilargi_embed_grad``, the layers through ``ilargi_linear`` and ``ilargi_linear_grad``, and the square
matrix W1 is updated by ``ilargi_orthogonalize``, the others by momentum.

    python examples/train_hidden_layer.py [--rows 200000] [--width 64] [--steps 30]
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


class HiddenLayerModel:
    """The weights, and the buffers that its steps keep."""

    def __init__(self, plan, fk, table_rows, width, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
        self.plan, self.fk, self.n, self.width, self.scale = plan, fk, plan.r_T, width, math.sqrt(width)
        self.weights = {"W0": new(plan.c_T, width) / math.sqrt(plan.c_T), "E": new(table_rows, width) * 0.1 / self.scale,
                        "W1": new(width, width) / math.sqrt(width), "b1": torch.zeros(width, device="cuda"),
                        "w2": new(width, 1) / math.sqrt(width), "b2": torch.zeros(1, device="cuda")}
        self.momentum = {k: torch.zeros_like(w) for k, w in self.weights.items()}
        rows = lambda m: torch.empty(self.n, m, device="cuda")
        self.H, self.pre1, self.H1, self.z, self.p = rows(width), rows(width), rows(width), rows(1), rows(1)
        layers = [il.ilargi_linear_workspace_bytes(self.n, width, m, torch.float32) for m in (width, 1)]
        nbytes = max(max(max(b) for b in layers), il.ilargi_embed_grad_workspace_bytes(self.n, table_rows, width),
                     il.ilargi_orthogonalize_workspace_bytes(1, width, width, torch.float32))
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")

    def forward(self):
        w, ws = self.weights, self.workspace
        il.ilargi_lmm(self.plan, w["W0"], out=self.H)
        il.ilargi_embed(w["E"], self.fk, self.scale, out=self.H, accumulate=True)
        il.ilargi_linear(self.H, w["W1"], bias=w["b1"], residual=self.H, act="gelu", out=self.H1, pre=self.pre1, workspace=ws)
        il.ilargi_linear(self.H1, w["w2"], bias=w["b2"], act="sigmoid", out=self.p, pre=self.z, workspace=ws)
        return self.p

    def loss(self, y):
        z = self.z[:, 0].double()
        return float((torch.nn.functional.softplus(z) - y * z).mean())

    def gradients(self, y):
        """Of the mean cross entropy, after ``forward``: its gradient by z is (p - y) / n."""
        w, ws = self.weights, self.workspace
        d_z = (self.p - y[:, None]) / self.n
        d_H1, d_w2, d_b2 = il.ilargi_linear_grad(d_z, self.H1, w["w2"], workspace=ws)
        d_H, d_W1, d_b1 = il.ilargi_linear_grad(d_H1, self.H, w["W1"], pre=self.pre1, act="gelu", workspace=ws)
        d_H += d_H1                                    # the residual's share
        d_E = il.ilargi_embed_grad(d_H, self.fk, w["E"].shape[0], self.scale, workspace=ws)
        return {"W0": il.ilargi_tmm(self.plan, d_H), "E": d_E, "W1": d_W1, "b1": d_b1, "w2": d_w2, "b2": d_b2}

    def step(self, y, lr, lr_square, beta=0.9):
        self.forward()
        for k, g in self.gradients(y).items():
            m, w = self.momentum[k], self.weights[k]
            m.mul_(beta).add_(g)
            if k == "W1":
                il.ilargi_orthogonalize(g + beta * m, out=w, base=w, alpha=-lr_square, beta=1.0, workspace=self.workspace)
            else:
                w.sub_(m, alpha=lr)


def problem(rows, table_rows=1000, entity_cols=6, joined_cols=10, seed=0):
    """A star join whose labels depend on a hidden value of every row of the joined table, so that E has something to learn."""
    rng = datagen.rng_for(seed)
    schema = datagen.star_schema(rng, rows, entity_cols, [(table_rows, joined_cols, "uniform")])
    hidden = rng.standard_normal(table_rows)
    fk = schema.sources[1].row_idx
    logit = 2.0 * hidden[fk] + schema.sources[0].D[:, 0] * schema.sources[1].D[fk, 0]
    y = (rng.random(rows) < 1.0 / (1.0 + np.exp(-logit))).astype(np.float32)
    sources = il.schema_to_device(schema)
    return sources, sources[1][1], schema, torch.from_numpy(y).cuda()


def train(rows=200_000, width=64, steps=30, table_rows=1000, lr=0.5, lr_square=0.005, seed=0, report=None):
    """Returns the loss before every step and after the last, and the model."""
    sources, fk, schema, y = problem(rows, table_rows, seed=seed)
    plan = il.ilargi_plan_create(sources, schema.r_T, schema.c_T, max_cx=width)
    model = HiddenLayerModel(plan, fk, table_rows, width, seed)
    losses = []
    for k in range(steps):
        model.step(y, lr, lr_square)
        losses.append(model.loss(y))
        if report is not None:
            report(k, losses[-1])
    model.forward()
    losses.append(model.loss(y))
    return losses, model


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rows", type=int, default=200_000)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    losses, _ = train(a.rows, a.width, a.steps, report=lambda k, v: print(f"step {k}: loss {v:.4f}", flush=True))
    print(f"after {a.steps} steps: loss {losses[-1]:.4f}")
