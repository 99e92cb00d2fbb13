"""The norms, the layers by group and the clipping as a program uses them together (examples/train_grouped_blocks.py): gradients of the whole
model against 64 bits, and a training step captured into a graph."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import train_grouped_blocks as mod
    return mod


def _model(ex, rows, width, hidden, keys):
    sources, schema, y = ex.problem(rows, keys)
    plan = ex.il.ilargi_plan_create(sources, schema.r_T, schema.c_T, max_cx=width)
    model = ex.GroupedBlockModel(plan, width, hidden)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for k in ("gain1", "gain2", "gate", "gain3", "b1", "b"):
        w = model.weights[k]
        w.add_(torch.randn(w.shape, generator=gen, device="cuda") * 0.3)
    return model, y[model.perm.long()]


def _loss64(ex, model, w, y):
    T = ex.il.ilargi_materialize(model.plan)[model.perm.long()].double()
    unit = lambda v: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6)
    key = torch.repeat_interleave(torch.arange(model.starts.numel() - 1, device="cuda"), (model.starts[1:] - model.starts[:-1]).long())
    H = T @ w["W0"]
    Y = unit(H) * w["gain1"]
    O = torch.zeros_like(H)
    for g in range(model.starts.numel() - 1):
        rows = key == g
        O = O.index_add(0, rows.nonzero()[:, 0], torch.nn.functional.silu(Y[rows] @ w["W1"][g] + w["b1"][g]) @ w["W2"][g])
    Z = unit(H + w["gate"] * unit(O) * w["gain2"]) * w["gain3"]
    z = (Z @ w["w"] + w["b"])[:, 0]
    return (torch.nn.functional.softplus(z) - y.double() * z).mean()


@pytest.mark.parametrize("rows,width,hidden,keys", [(500, 12, 20, 5), (4000, 33, 48, 70)])
def test_gradients(ex, rows, width, hidden, keys):
    """float32 through eight operators in a row: each is good to a few 2^-24 of its results' size (their own tests have the bounds), so the
    gradients, sums over the rows, agree to 2e-5 of their norm: 300 roundings."""
    model, y = _model(ex, rows, width, hidden, keys)
    model.forward()
    grads = model.gradients(y)
    w = {k: v.double().requires_grad_(True) for k, v in model.weights.items()}
    loss = _loss64(ex, model, w, y)
    assert abs(model.loss(y) - float(loss)) <= 1e-6 * (1 + float(loss))
    want = torch.autograd.grad(loss, list(w.values()))
    for (k, g), v in zip(grads.items(), want):
        assert float((g.double() - v).norm()) <= 2e-5 * float(v.norm()) + 1e-12, k


def test_steps_run_and_stay_below_the_largest_norm(ex):
    losses, model = ex.train(rows=3000, width=16, hidden=24, keys=7, steps=4, max_norm=0.05)
    assert all(v == v and v < 10 for v in losses)
    total = sum(float(g.double().square().sum()) for g in model.grads.values()) ** 0.5
    assert total <= 0.05 * (1 + 1e-6)


def test_step_in_a_graph(ex):
    model, y = _model(ex, 2000, 24, 40, 9)
    state = {k: w.clone() for k, w in model.weights.items()}
    model.step(y, 0.1, 0.1)                                   # outside of the graph first: buffers of torch's are made
    want = {k: w.clone() for k, w in model.weights.items()}
    for k, w in model.weights.items():
        w.copy_(state[k])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        model.step(y, 0.1, 0.1)
    for _ in range(3):
        for k, w in model.weights.items():
            w.copy_(state[k])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(w, want[k]) for k, w in model.weights.items())
