"""Attention and embedding gradients keep states, keys and sums in their workspaces, where calls of other kinds and sizes keep the status words of their chains:
what finds such a workspace clears its status words first (no GPU; addresses are never followed)."""
import pytest

import launch_recorder
from operator_launches import launches, shape
from paper_2411_17887_amd import tcuscan

AT = [0x100000 * (i + 1) for i in range(12)]
WS, OTHER, BYTES = 0x10000 + (1 << 36), 0x10000 + (1 << 37), 1 << 32


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    shim = launch_recorder.build(tmp_path_factory.mktemp("shim"))
    return lambda calls: launches(shim, calls)


def scan(ws=WS, n=1 << 20):
    return ("tcuscan_inclusive", [AT[0], AT[1], n, tcuscan.I32_I32, ws, BYTES, 0])


def gradient(n, ws=WS, dim=16):
    return ("tcuscan_embedding_backward", [AT[0], 8, n, AT[1], dim, tcuscan.BF16_F32, AT[2], 900, dim, dim, tcuscan.F32_F32, -1, 0, ws, BYTES, 0])


def prompt(total, ws=WS):
    return ("tcuscan_decay_attention", [shape(1, total, 4, 64, 64), *AT[:6], tcuscan.BF16_F32, 0, 0, 0, 0, ws, BYTES, 0])


def backward(total, ws=WS, k=4):
    return ("tcuscan_decay_attention_backward", [shape(1, total, 4, 64, 64, k=k), *AT[:9], tcuscan.F32_F32, 0, 0, 0, ws, BYTES, 0])


def cleared(result):
    """Whether something clears words in front of the call's scan or split kernels."""
    rc, kernels = result
    assert rc == tcuscan.OK
    names = [k[0] for k in kernels]
    chain = [i for i, n in enumerate(names) if n.startswith(("scan_kernel<", "split_kernel<"))]
    assert chain
    return any(n == "fill_zero_kernel" for n in names[max(0, chain[0] - 1):chain[0]])


@pytest.mark.parametrize("first", [gradient(9000), prompt(5000), backward(5000), backward(100, k=2)], ids=["embedding", "prompt", "gradients", "parts"])
def test_a_scan_clears_what_operators_on_tokens_left(run, first):
    got = run([scan(), first, scan(), scan(), scan(OTHER)])
    assert [cleared(got[i]) for i in (0, 2, 3, 4)] == [False, True, False, False]


@pytest.mark.parametrize("first", [prompt(200), backward(200), gradient(4096)], ids=["prompt", "gradients", "embedding"])
def test_calls_that_keep_nothing_cost_no_clearing(run, first):
    got = run([scan(), first, scan()])
    assert not cleared(got[0]) and not cleared(got[2])


@pytest.mark.parametrize("form", [0, 2])
def test_sorts_with_a_chain_clear_the_keys_of_a_smaller_call(run, form):
    """The sorted keys of 9000 tokens lie where those of a million have status words; so do a call's own sums."""
    got = run([("tcuscan_set_sort_fusion", [form]), gradient(1_000_000), gradient(9000), gradient(1_000_000), gradient(40_000), gradient(1_000_000)])
    assert all(cleared(got[i]) for i in (1, 3, 4, 5))          # (9000 pairs are one tile in form 2: no chain)
    assert got[2][0] == tcuscan.OK
