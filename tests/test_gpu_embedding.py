"""Rows of an embedding table and the table's gradient by sorted tokens, on the GPU, against the definition in 64 bits."""
import numpy as np
import pytest

from paper_2411_17887_amd import tcuscan

pytestmark = pytest.mark.gpu

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
SUBNORMAL = {"bf16": 0.0, "f16": 2.0 ** -25, "f32": 0.0}
KINDS = ["bf16", "f16", "f32"]


def torch_kind(kind):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[kind]


def table(rows, dim, kind, seed, pad=0):
    """Values on the GPU, `pad` unused elements behind every row, and the same in 64 bits."""
    import torch
    x = torch.randn(rows, dim + pad, generator=torch.Generator().manual_seed(seed)).to(torch_kind(kind))
    return x.cuda()[:, :dim], x[:, :dim].double().numpy()


def check_lookup(ids, vocab, dim, w_kind, o_kind, scale=3.7, pad=0, id_type=np.int64):
    import torch
    weight, host = table(vocab, dim, w_kind, 1, pad)
    ids = np.asarray(ids, dtype=id_type)
    guard = torch.full((len(ids) + 2, dim + pad), -77.0, dtype=torch_kind(o_kind), device="cuda")
    out = guard[1:-1, :dim]
    tcuscan.embedding(torch.from_numpy(ids).cuda(), weight, out, scale=scale)
    torch.cuda.synchronize()
    there = (ids >= 0) & (ids < vocab)
    want = np.where(there[:, None], host[np.where(there, ids, 0)] * np.float64(np.float32(scale)), 0.0)
    # two roundings: the product in fp32, the output
    assert (np.abs(out.double().cpu().numpy() - want) <= (UNIT[o_kind] + 2.0 ** -24) * np.abs(want) + SUBNORMAL[o_kind]).all()
    assert (guard[0] == -77.0).all() and (guard[-1] == -77.0).all() and (guard[:, dim:] == -77.0).all()


@pytest.mark.parametrize("w_kind", KINDS)
@pytest.mark.parametrize("o_kind", KINDS)
def test_lookup_in_all_types(w_kind, o_kind):
    rng = np.random.RandomState(1)
    check_lookup(rng.randint(0, 300, 500), 300, 136, w_kind, o_kind)


@pytest.mark.parametrize("dim", [1, 2, 7, 8, 64, 65, 200, 512, 1000, 4096, 5001])
@pytest.mark.parametrize("n", [1, 3, 130])
def test_lookup_of_all_sizes(n, dim):
    rng = np.random.RandomState(2)
    for pad in (0, 1, 8):
        check_lookup(rng.randint(0, 50, n), 50, dim, "bf16", "bf16", pad=pad)
        check_lookup(rng.randint(0, 50, n), 50, dim, "f32", "f16", pad=pad, id_type=np.int32)


def test_lookup_of_no_token_and_numbers_out_of_range():
    import torch
    check_lookup([-1, 3, -(1 << 40), 0, 9], 10, 24, "f32", "bf16")
    weight, _ = table(10, 24, "f32", 1)
    ws = torch.zeros(32, dtype=torch.int64, device="cuda")
    out = torch.full((3, 24), -77.0, device="cuda")
    tcuscan.embedding(torch.tensor([1, 10, 1 << 40]).cuda(), weight, out, ws=ws)
    torch.cuda.synchronize()
    assert tcuscan.workspace_fault(ws) == 2 and torch.equal(out[0], weight[1]) and (out[1:] == 0).all()
    tcuscan.embedding(torch.empty(0, dtype=torch.int64, device="cuda"), weight, out[:0])


def zipf(n, vocab, seed):
    r = np.random.RandomState(seed)
    p = 1.0 / (np.arange(vocab) + 2.0)
    return r.permutation(vocab)[r.choice(vocab, n, p=p / p.sum())]


def check_gradient(ids, vocab, dim, g_kind="f32", w_kind="f32", scale=0.7, padding=-1, accumulate=False, pad=0, id_type=np.int64, ws=None):
    import torch
    ids = np.asarray(ids, dtype=id_type)
    n = len(ids)
    d_out, host = table(n, dim, g_kind, 3, pad)
    before, old = table(vocab, dim, w_kind, 4, pad)
    guard = torch.full((vocab + 2, dim + pad), -77.0, dtype=torch_kind(w_kind), device="cuda")
    d_weight = guard[1:-1, :dim]
    d_weight.copy_(before)
    ws = tcuscan.new_embedding_backward_workspace(n, vocab, dim) if ws is None else ws
    runs = []
    for _ in range(2):
        d_weight.copy_(before)
        tcuscan.embedding_backward(torch.from_numpy(ids).cuda(), d_out, d_weight, scale=scale, padding=padding, accumulate=accumulate, ws=ws)
        torch.cuda.synchronize()
        runs.append(d_weight.clone())
    assert tcuscan.workspace_fault(ws) == 0
    assert torch.equal(runs[0], runs[1])
    assert (guard[0] == -77.0).all() and (guard[-1] == -77.0).all() and (guard[:, dim:] == -77.0).all()
    counted = (ids >= 0) & (ids != padding)
    want, size, counts = np.zeros((vocab, dim)), np.zeros((vocab, dim)), np.bincount(ids[counted], minlength=vocab)
    np.add.at(want, ids[counted], host[counted])
    np.add.at(size, ids[counted], np.abs(host[counted]))
    scale = np.float64(np.float32(scale))
    want, size = want * scale, size * abs(scale)
    if accumulate:
        want, size = want + old, size + np.abs(old)
    got = runs[0].double().cpu().numpy()
    # one fp32 rounding for each addition of a row's tokens, for the scale and for what was there; the table's own rounding at the end
    bound = UNIT[w_kind] * np.abs(want) + (counts[:, None] + 2.0) * 2.0 ** -24 * size * (1 + UNIT[w_kind]) + SUBNORMAL[w_kind]
    assert (np.abs(got - want) <= bound).all()
    if accumulate:
        untouched = counts == 0
        assert np.array_equal(got[untouched], old[untouched])


@pytest.mark.parametrize("g_kind", KINDS)
@pytest.mark.parametrize("w_kind", KINDS)
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_in_all_types(g_kind, w_kind, accumulate):
    check_gradient(zipf(3000, 400, 5), 400, 136, g_kind, w_kind, accumulate=accumulate)


@pytest.mark.parametrize("dim", [1, 3, 8, 65, 515, 1024, 4100])
@pytest.mark.parametrize("n,vocab", [(0, 7), (1, 1), (1, 900), (70, 3), (700, 2000), (4097, 50)])
def test_gradient_of_all_sizes(n, vocab, dim):
    for pad in (0, 1):
        check_gradient(zipf(n, vocab, 6), vocab, dim, "bf16", "f32", pad=pad, accumulate=pad == 1, id_type=np.int32 if pad else np.int64)


@pytest.mark.parametrize("ids", [[5] * 5000, [0] * 31 + [1] * 33 + [2] * 64 + [3] * 1, list(range(600)) * 3, [7] * 700 + [8] + [9] * 700, [599] * 100 + [0] * 2000], ids=["one", "blocks", "all", "two", "ends"])
def test_gradient_of_long_runs(ids):
    """Runs of one token number that begin and end inside, at and across the pieces they are summed in."""
    check_gradient(np.random.RandomState(7).permutation(ids), 600, 72)
    check_gradient(ids, 600, 72, "f16", "bf16", accumulate=True)


def test_gradient_of_a_large_table_and_many_tokens():
    check_gradient(zipf(40_000, 70_000, 8), 70_000, 40, "bf16", "f32")


def test_padding_and_numbers_out_of_range():
    import torch
    ids = zipf(2000, 100, 9)
    common = int(np.bincount(ids).argmax())
    check_gradient(ids, 100, 48, padding=common)
    check_gradient(np.where(ids % 5 == 0, -3, ids), 100, 48)
    check_gradient([-1] * 90, 100, 48)
    ws = tcuscan.new_embedding_backward_workspace(3, 10, 8)
    d_weight = torch.full((10, 8), -77.0, device="cuda")
    tcuscan.embedding_backward(torch.tensor([1, 10, 1 << 35]).cuda(), torch.ones(3, 8, device="cuda"), d_weight, ws=ws)
    torch.cuda.synchronize()
    assert tcuscan.workspace_fault(ws) == 2
    want = torch.zeros(10, 8)
    want[1] = 1.0
    assert torch.equal(d_weight.cpu(), want)


def test_gradient_against_differences():
    """<d_out, out> is linear in the table: its difference along any direction is <d_weight, direction>."""
    import torch
    ids = zipf(800, 60, 10)
    d_out, host = table(800, 33, "f32", 3)
    ws = tcuscan.new_embedding_backward_workspace(800, 60, 33)
    d_weight = torch.empty(60, 33, device="cuda")
    dev_ids = torch.from_numpy(ids).cuda()
    tcuscan.embedding_backward(dev_ids, d_out, d_weight, scale=2.5, ws=ws)
    along, along_host = table(60, 33, "f32", 11)
    out = torch.empty(800, 33, device="cuda")
    tcuscan.embedding(dev_ids, along, out, scale=2.5)
    torch.cuda.synchronize()
    left, right = (out.double().cpu().numpy() * host).sum(), (d_weight.double().cpu().numpy() * along_host).sum()
    size = np.abs(out.double().cpu().numpy() * host).sum()
    assert abs(left - right) <= (np.bincount(ids).max() + 3) * 2.0 ** -24 * size


def test_one_workspace_for_calls_of_different_sizes_and_sorts():
    ws = tcuscan.new_embedding_backward_workspace(30_000, 900, 16)
    for form in (1, 2, 0, 1):
        tcuscan.set_sort_fusion(form)
        try:
            check_gradient(zipf(30_000, 900, 12), 900, 16, ws=ws)
            check_gradient(zipf(50, 300, 13), 300, 16, ws=ws)
            check_gradient(zipf(9000, 5000, 14), 5000, 16, ws=ws)
        finally:
            tcuscan.set_sort_fusion(1)


def test_gradient_in_a_graph():
    import torch
    ids, d_out = torch.from_numpy(zipf(20_000, 500, 15)).cuda(), table(20_000, 64, "bf16", 16)[0]
    ws, d_weight = tcuscan.new_embedding_backward_workspace(20_000, 500, 64), torch.empty(500, 64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    tcuscan.embedding_backward(ids, d_out, d_weight, ws=ws, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tcuscan.embedding_backward(ids, d_out, d_weight, ws=ws, stream=side)
    other, eager = tcuscan.new_embedding_backward_workspace(20_000, 500, 64), torch.empty_like(d_weight)
    for rep in range(4):
        ids.copy_(torch.from_numpy(zipf(20_000, 500, 20 + rep)))
        d_weight.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        tcuscan.embedding_backward(ids, d_out, eager, ws=other)
        torch.cuda.synchronize()
        assert torch.equal(d_weight, eager)


def test_rows_further_apart_than_32_bits_reach():
    """A table and a gradient of more than 2^32 bytes."""
    import torch
    vocab, dim = 1_100_000, 2048
    weight = torch.empty(vocab, dim, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([0, vocab - 1, vocab // 2, vocab - 1])
    rows = torch.randn(4, dim, generator=torch.Generator().manual_seed(1)).bfloat16()
    rows[3] = rows[1]
    weight[ids.cuda()] = rows.cuda()
    out = torch.empty(4, dim, dtype=torch.bfloat16, device="cuda")
    tcuscan.embedding(ids.cuda(), weight, out)
    ws = tcuscan.new_embedding_backward_workspace(4, vocab, dim)
    tcuscan.embedding_backward(ids.cuda(), out, weight, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), rows)
    want = {0: rows[0], vocab // 2: rows[2], vocab - 1: (rows[1].float() * 2).bfloat16()}
    for r, w in want.items():
        assert torch.equal(weight[r].cpu(), w)
    assert int((weight != 0).any(1).sum()) == 3


@pytest.mark.parametrize("n", [4095, 4096, 4097, 4160])
def test_gradient_on_both_sides_of_the_choice_of_form(n):
    check_gradient(zipf(n, 3000, 30 + n), 3000, 24, "bf16", "f32")
    check_gradient([11] * n, 64, 40, "f16", "f16", accumulate=True)


@pytest.mark.parametrize("w_kind", KINDS)
@pytest.mark.parametrize("dim", [1, 7, 9, 31, 513, 530])
def test_rows_of_no_token_start_and_end_anywhere(dim, w_kind):
    """Most rows are cleared 16 bytes at a time; they start and end at every element within 16 bytes."""
    for pad in (0, 1, 3):
        check_gradient([3, 40, 40, 199], 200, dim, "bf16", w_kind, pad=pad)


@pytest.mark.parametrize("ids", [[4] * 4096, [4, 9] * 2048, [i % 8 for i in range(4096)], [1] * 512 + [2] * 1500 + [1] * 2, [3] * 513], ids=["one", "two", "eight", "shares", "edge"])
def test_few_tokens_with_numbers_that_many_share(ids):
    check_gradient(ids, 70, 72)
    check_gradient(ids, 70, 19, "bf16", "f16", accumulate=True)
