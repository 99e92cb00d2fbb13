"""The example that trains learned features over a join: its gradients against 64 bits, and that it learns."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_hidden_layer.py")
    spec = importlib.util.spec_from_file_location("train_hidden_layer", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("rows,width", [(3001, 17), (4096, 64)])
def test_gradients_against_64_bits(example, rows, width):
    """float32 sums of n terms: relative errors of about sqrt(n) 2^-24 a product, five in a row; 1e-5 leaves a margin of ten."""
    il = example.il
    sources, fk, schema, y = example.problem(rows, 50, seed=3)
    plan = il.ilargi_plan_create(sources, schema.r_T, schema.c_T, max_cx=width)
    model = example.HiddenLayerModel(plan, fk, 50, width, seed=1)
    model.forward()
    got = model.gradients(y)
    w = {k: v.double().requires_grad_() for k, v in model.weights.items()}
    T = il.ilargi_materialize(plan).double()
    H = T @ w["W0"] + model.scale * w["E"][fk.long()]
    H1 = torch.nn.functional.gelu(H @ w["W1"] + w["b1"]) + H
    z = (H1 @ w["w2"] + w["b2"])[:, 0]
    loss = (torch.nn.functional.softplus(z) - y.double() * z).mean()
    loss.backward()
    assert abs(model.loss(y) - float(loss.detach())) <= 1e-5
    for k, g in got.items():
        want = w[k].grad
        assert float((g.double() - want).norm()) <= 1e-5 * float(want.norm()), k


def test_it_learns(example):
    losses, model = example.train(rows=20_000, width=32, steps=25, table_rows=200)
    assert losses[-1] < 0.85 * losses[0] and all(bool(torch.isfinite(w).all()) for w in model.weights.values())
    again, _ = example.train(rows=20_000, width=32, steps=25, table_rows=200)
    assert losses == again
