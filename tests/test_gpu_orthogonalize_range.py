"""Orthogonalised updates over the whole range of norms, eps, steps and sizes of the parts of G, against 64 bits.

A step's products are good to e = 3 (sqrt(l) + 4) u32 of its result, as in the tests at ordinary norms: after T steps the result is off
by at most e (a^T - 1) / (a - 1) of the norm that unamplified directions have.  Where all singular values are small, the whole result
is such a direction, and T e of it bounds the error; the first is larger for every T here.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16
COEF = (3.4445, -4.7750, 2.0315)
U32 = 2.0 ** -24


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


def _tol(rows, cols, steps, out=F32):
    a = COEF[0]
    return 3 * (math.sqrt(max(rows, cols)) + 4) * U32 * (a ** steps - 1) / (a - 1) + (2.0 ** -8 if out == BF16 else 0.0)


def _far(got, want):
    return float((got.double() - want).norm() / want.norm())


def _of_norm(shape, norm, gen):
    G = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float64)
    return (G * (norm / G.square().sum((-1, -2), keepdim=True).sqrt())).float()


# one workgroup's matrices, general ones, tall ones
@pytest.mark.parametrize("shape", [(64, 220), (220, 60), (600, 700), (1030, 300)])
@pytest.mark.parametrize("norm", [1e-37, 1e-36, 1e-33, 1e38, 3e40])
def test_norms_at_the_ends_of_float32(il, shape, norm):
    """eps = 0: the result does not depend on the norm, though 1 / norm, or the norm itself, is no float32 number."""
    if norm > 1e39 and shape[0] * shape[1] < 300_000:
        pytest.skip("entries would be infinite")
    G = _of_norm((1, *shape), norm, _gen(shape[0]))
    assert bool(torch.isfinite(G).all())
    for steps in (1, 5):
        assert _far(il.ilargi_orthogonalize(G, steps=steps, eps=0.0), _exact(G, steps, eps=0.0)) <= _tol(*shape, steps)
