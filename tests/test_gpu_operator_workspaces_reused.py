"""A workspace that embedding gradients have used is fit for scans and for sorts with a chain, although sorted token numbers lie where status words do and
can look like those of an early call."""
import numpy as np
import pytest

from test_gpu_embedding import check_gradient, zipf
from paper_2411_17887_amd import tcuscan

pytestmark = pytest.mark.gpu


def test_scans_after_embedding_gradients():
    import torch
    n = 1 << 20
    ws = torch.zeros(max(tcuscan.workspace_bytes(1, n, "i32"), tcuscan.embedding_backward_workspace_bytes(60_000, 1 << 22, 8)) // 8 + 1, dtype=torch.int64, device="cuda")
    x, out = torch.ones(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    want = torch.arange(1, n + 1, dtype=torch.int32, device="cuda")
    for base in (0, 40, 400, 4000):                            # (a status word's high half is four times its call's number, and more)
        ids = base + torch.arange(60_000, device="cuda") // 3
        d_weight = torch.empty(1 << 22, 8, device="cuda")
        tcuscan.embedding_backward(ids, torch.ones(60_000, 8, device="cuda"), d_weight, ws=ws)
        tcuscan.inclusive(x, out, "i32", ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and tcuscan.workspace_fault(ws) == 0


@pytest.mark.parametrize("form", [0, 2])
def test_sorts_with_a_chain_after_smaller_calls(form):
    ws = tcuscan.new_embedding_backward_workspace(300_000, 30_000, 8)
    tcuscan.set_sort_fusion(form)
    try:
        for n, vocab in ((9000, 3000), (300_000, 30_000), (9000, 30_000), (70_000, 5000), (300_000, 30_000)):
            check_gradient(np.sort(zipf(n, vocab, n)), vocab, 8, ws=ws)
    finally:
        tcuscan.set_sort_fusion(1)
