"""Workspaces of the layers that need no GPU: what a call cannot use is not asked for."""
import pytest

torch = pytest.importorskip("torch")

import paper_2502_01985_amd as il  # noqa: E402


@pytest.mark.parametrize("n,k,m", [(1, 32768, 32768), (2, 8192, 8192), (1, 4096, 262144)])
def test_few_rows_ask_for_sums_only(n, k, m):
    """Up to two rows of bfloat16 read W where it lies: at most a share of k for every 1024 of it, m floats a row each."""
    assert il.ilargi_linear_workspace_bytes(n, k, m, torch.bfloat16)[0] <= (k // 1024) * n * m * 4 + 256


def test_rows_that_are_laid_out_ask_for_the_copies():
    """X and W of rows that end inside 16 bytes are copied where the product is worth it."""
    n, k, m = 2001, 701, 603
    assert il.ilargi_linear_workspace_bytes(n, k, m, torch.bfloat16)[0] >= 2 * (n * 704 + k * 608)
