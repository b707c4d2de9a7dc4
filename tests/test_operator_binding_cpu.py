"""Token numbers that are no integers (no GPU)."""
import pytest

from paper_2411_17887_amd import tcuscan


def test_complex_token_numbers_are_refused():
    torch = pytest.importorskip("torch")
    ids, table, rows = torch.zeros(3, dtype=torch.complex64), torch.zeros(9, 5), torch.zeros(3, 5)     # 8 bytes each, and no floating-point type to torch
    with pytest.raises(ValueError):
        tcuscan.embedding(ids, table, rows)
    with pytest.raises(ValueError):
        tcuscan.embedding_backward(ids, rows, table)
