"""The squares' order depends on the inputs alone: what is written, and where to, leaves the norm's bits as they are.

The entries tell orders apart in float32: 1, 2^-12 twice and 2^-24 have squares of (1 + 2^-24)^2 together, whose root lies between two float32
numbers.  Nine entries with squares just below 2^-53 are lost one by one where they follow those in a thread's sum, and together carry the root
over where they have threads of their own.  The norm is one or the other, and has to be the same one.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def il():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_01985_amd as mod
    return mod


def test_outputs_do_not_change_the_norm(il):
    t = torch.zeros(4, 1025, device="cuda")
    flat = t.view(-1)
    flat[:4] = torch.tensor([1.0, 2.0 ** -12, 2.0 ** -12, 2.0 ** -24], device="cuda")
    for at in (1025, 1026, 1027, 2049, 2050, 2051, 3073, 3074, 3075):
        flat[at] = 1.4 * 2.0 ** -27
    padded = torch.empty(4, 1030, device="cuda")[:, :1025]
    norms = [il.ilargi_clip_norm(il.TensorList([t], outs), math.inf) for outs in (None, [torch.empty_like(t)], [padded], [t])]
    assert float(norms[0]) in (1.0, 1.0 + 2.0 ** -23)
    assert all(torch.equal(norms[0], v) for v in norms[1:])
    assert torch.equal(padded, t)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_padded_outputs_of_some_tensors(il, dtype):
    """Passes over inputs and outputs that are cut differently: scaled as in place, by the same norm; rows behind the outputs' columns stay."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    shapes = [(300, 333), (7, 5), (1, 9), (2100, 1031), (64, 64), (40, 3)] * 12
    tensors = [torch.randn(s, generator=gen, device="cuda").to(dtype) for s in shapes]
    wide = [torch.full((s[0], s[1] + 3), 7.0, dtype=dtype, device="cuda") for s in shapes]
    outs = [w[:, : s[1]] if q % 3 else None for q, (w, s) in enumerate(zip(wide, shapes))]
    norm = il.ilargi_clip_norm(il.TensorList(tensors), 1.0)
    assert torch.equal(il.ilargi_clip_norm(il.TensorList(tensors, outs), 1.0), norm)
    inplace = [t.clone() for t in tensors]
    assert torch.equal(il.ilargi_clip_norm(inplace, 1.0), norm)
    for q, (o, w, i, s) in enumerate(zip(outs, wide, inplace, shapes)):
        assert o is None or torch.equal(o, i)
        assert bool((w[:, s[1] if o is not None else 0:] == 7).all())
