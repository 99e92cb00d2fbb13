"""Empty tensors of the clipping that have rows but no columns: nothing is read or written of them, whatever their leading dimensions."""
import ctypes

import pytest

import paper_2502_01985_amd as il


@pytest.mark.parametrize("rows,cols,ld_in,ld_out", [(5, 0, 7, 0), (5, 0, 0, 3), (0, 4, 4, 9)])
def test_an_empty_tensor_without_addresses(rows, cols, ld_in, ld_out):
    entry = il.TensorStruct(None, None, rows, cols, ld_in, ld_out, 0)
    nbytes = ctypes.c_size_t()
    assert il.lib.ilargi_clip_norm_workspace_bytes((il.TensorStruct * 1)(entry), 1, ctypes.byref(nbytes)) == il.OK
    assert nbytes.value >= 8


def test_in_place_with_another_leading_dimension_stays_refused():
    entry = il.TensorStruct(1 << 20, 1 << 20, 4, 8, 8, 9, 0)
    nbytes = ctypes.c_size_t()
    assert il.lib.ilargi_clip_norm_workspace_bytes((il.TensorStruct * 1)(entry), 1, ctypes.byref(nbytes)) == il.ERR_SHAPE
