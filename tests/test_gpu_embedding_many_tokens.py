"""The table's gradient of more tokens than one launch takes: numbers that add nothing (padding, negative, not below the table's height) sort behind all rows,
in runs that begin and end inside and across the pieces that runs are summed in."""
import numpy as np
import pytest

from test_gpu_embedding import KINDS, check_gradient, table, zipf
from paper_2411_17887_amd import tcuscan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [4097, 6000, 20_011])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("id_type", [np.int32, np.int64])
def test_padding_and_negative_numbers(n, accumulate, id_type):
    ids = zipf(n, 300, n)
    common, rare = int(np.bincount(ids).argmax()), int(np.bincount(ids, minlength=300).argmin())
    for padding in (common, rare, 0, 299, -100, 300):
        check_gradient(ids, 300, 40, "bf16", "f32", padding=padding, accumulate=accumulate, id_type=id_type)
    check_gradient(np.where(np.arange(n) % 3 == 0, -1, ids), 300, 40, accumulate=accumulate, id_type=id_type)
    check_gradient(np.where(ids == common, -(1 << 31), ids), 300, 33, "f16", "f16", padding=rare, accumulate=accumulate, id_type=id_type)


@pytest.mark.parametrize("kind", KINDS)
def test_no_token_counts(kind):
    for ids, padding in ((np.full(5000, -1), -1), (np.full(4500, 7), 7), (np.arange(9000) % 2 - 1, 0)):
        check_gradient(ids, 100, 24, kind, kind, padding=padding)
        check_gradient(ids, 100, 24, kind, kind, padding=padding, accumulate=True)


@pytest.mark.parametrize("counts", [31, 32, 33, 64, 4000])
def test_a_run_of_nothing_behind_the_last_row(counts):
    """The last row's run ends, and the run of numbers that add nothing begins, at and around the ends of pieces."""
    n = 4100 + counts
    ids = np.concatenate([np.arange(n - counts - 70) % 299, np.full(70, 299), np.full(counts, -2)])
    check_gradient(np.random.RandomState(61).permutation(ids), 300, 72, "bf16", "bf16")


@pytest.mark.parametrize("form", [0, 1, 2])
@pytest.mark.parametrize("accumulate", [False, True])
def test_numbers_out_of_range_are_reported_and_add_nothing(form, accumulate):
    import torch
    n, vocab, dim = 6000, 200, 24
    ids = zipf(n, vocab, 62).astype(np.int64)
    bad = np.random.RandomState(63).rand(n) < 0.2
    wrong = np.where(bad, np.where(np.arange(n) % 2 == 0, vocab, 1 << 40), ids)
    d_out, host = table(n, dim, "f32", 64)
    guard = torch.full((vocab + 2, dim), -77.0, device="cuda")
    d_weight = guard[1:-1]
    d_weight.fill_(1.0 if accumulate else -77.0)
    ws = tcuscan.new_embedding_backward_workspace(n, vocab, dim)
    tcuscan.set_sort_fusion(form)
    try:
        tcuscan.embedding_backward(torch.from_numpy(wrong).cuda(), d_out, d_weight, accumulate=accumulate, ws=ws)
    finally:
        tcuscan.set_sort_fusion(1)
    torch.cuda.synchronize()
    assert tcuscan.workspace_fault(ws) == 2
    assert (guard[0] == -77.0).all() and (guard[-1] == -77.0).all()
    want, size = np.zeros((vocab, dim)), np.zeros((vocab, dim))
    np.add.at(want, ids[~bad], host[~bad])
    np.add.at(size, ids[~bad], np.abs(host[~bad]))
    want += float(accumulate)
    # one fp32 rounding for each addition of a row's tokens, for what was there and for the result
    bound = (np.bincount(ids[~bad], minlength=vocab)[:, None] + 3.0) * 2.0 ** -24 * (size + float(accumulate))
    assert (np.abs(d_weight.double().cpu().numpy() - want) <= bound).all()


def test_values_that_are_not_finite_stay_with_their_row():
    """Also those of tokens that add nothing, which lie in the same pieces."""
    import torch
    n, vocab, dim = 5000, 100, 40
    ids = np.sort(zipf(n, vocab, 65))
    ids[ids == 3] = -1
    d_out, _ = table(n, dim, "bf16", 66)
    ws, d_weight = tcuscan.new_embedding_backward_workspace(n, vocab, dim), torch.empty(vocab, dim, device="cuda")
    tcuscan.embedding_backward(torch.from_numpy(ids).cuda(), d_out, d_weight, ws=ws)
    want = d_weight.clone()
    spoiled = int(np.bincount(ids[ids >= 0]).argmax())
    d_out = d_out.clone()
    d_out[torch.from_numpy(ids < 0).cuda()] = float("nan")
    d_out[int(np.nonzero(ids == spoiled)[0][5])] = float("inf")
    tcuscan.embedding_backward(torch.from_numpy(ids).cuda(), d_out, d_weight, ws=ws)
    torch.cuda.synchronize()
    others = [r for r in range(vocab) if r != spoiled]
    assert torch.equal(d_weight[others], want[others]) and torch.isinf(d_weight[spoiled]).all()
