"""Where the norm is stored: in an element of a tensor of the call it would be written while other workgroups read that, so it is refused."""
import pytest

import paper_2502_01985_amd as il

P, FAR = 1 << 20, 1 << 30


def _call(norm, *entries):
    array = (il.TensorStruct * max(len(entries), 1))(*(il.TensorStruct(*e) for e in entries))
    # (without a workspace what is not refused for its places is refused for that: nothing runs)
    return il.lib.ilargi_clip_norm(array, len(entries), 1.0, norm, None, 0, None)


@pytest.mark.parametrize("norm,entry", [
    (P, (P, P, 4, 8, 8, 8, 0)), (P + 124, (P, P, 4, 8, 8, 8, 0)), (P + 60, (P, None, 4, 8, 8, 0, 0)), (FAR + 8, (P, FAR, 4, 8, 8, 8, 0)),
    (P + 12, (P, P, 4, 8, 16, 16, 1)), (P + 32, (P, P, 4, 8, 16, 16, 1)), (P + 30, (P, P, 4, 8, 16, 16, 1)), (P + 14, (P, P, 1, 8, 8, 8, 1)),
])
def test_in_a_tensor(norm, entry):
    assert _call(norm, entry) == il.ERR_SHAPE
    assert "norm" in il.ilargi_last_error()


@pytest.mark.parametrize("norm,entry", [
    (None, (P, P, 4, 8, 8, 8, 0)), (P + 128, (P, P, 4, 8, 8, 8, 0)), (P - 4, (P, P, 4, 8, 8, 8, 0)), (P + 32, (P, P, 4, 8, 16, 16, 0)), (P + 60, (P, P, 4, 8, 16, 16, 0)),
    (P + 16, (P, P, 4, 8, 16, 16, 1)), (P + 28, (P, P, 4, 8, 16, 16, 1)), (P + 16, (P, P, 1, 8, 8, 8, 1)),
])
def test_beside_a_tensor_and_between_its_rows(norm, entry):
    assert _call(norm, entry) == il.ERR_NULL


def test_tensors_of_two_types_in_one_matrix():
    """Rows of 64 bytes: 32 of float32 and 32 of bfloat16, side by side; then one that begins in the other."""
    assert _call(None, (P, P, 4, 8, 16, 16, 0), (P + 32, P + 32, 4, 16, 32, 32, 1)) == il.ERR_NULL
    assert _call(None, (P, P, 4, 8, 16, 16, 0), (P + 30, P + 30, 4, 16, 32, 32, 1)) == il.ERR_SHAPE
    assert _call(None, (P, P, 4, 8, 16, 16, 0), (P + 32, P + 32, 4, 17, 32, 32, 1)) == il.ERR_SHAPE
