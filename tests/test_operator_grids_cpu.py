"""No launch of the operators on tokens asks for 2^32 threads or more, which HIP does not take: such calls are refused as a whole, before anything is enqueued (no
GPU; addresses are never followed)."""
import pytest

import launch_recorder
from operator_launches import launches, shape
from paper_2411_17887_amd import tcuscan

AT = [0x100000 * (i + 1) for i in range(12)]
WS, BYTES = 1 << 44, 1 << 60
BF16, F32 = tcuscan.BF16_F32, tcuscan.F32_F32


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    shim = launch_recorder.build(tmp_path_factory.mktemp("shim"))
    return lambda calls: launches(shim, calls)


def prompt(s):
    return ("tcuscan_decay_attention", [s, *AT[:6], BF16, AT[6], AT[7], 0, 1 << 40, WS, BYTES, 0])


def backward(s):
    return ("tcuscan_decay_attention_backward", [s, *AT[:9], BF16, 0, 0, AT[9], WS, BYTES, 0])


def step(s):
    return ("tcuscan_decay_attention_step", [s, *AT[:5], BF16, AT[6], 0, 1 << 40, 0, 0, 0])


def lookup(n, dim, out=AT[2]):
    return ("tcuscan_embedding", [AT[0], 8, n, AT[1], 1000, dim, dim, BF16, out, dim, BF16, 0, 0, 0])


def gradient(n, vocab, dim, flags=0):
    return ("tcuscan_embedding_backward", [AT[0], 8, n, AT[1], dim, BF16, AT[2], vocab, dim, dim, F32, -1, flags, WS, BYTES, 0])


# (call, whether it fits), next to each other on both sides of a limit: 2^32 / 256 = 16777216 workgroups of 256 threads
CASES = {
    "rows": [(prompt(shape((1 << 20) - 1, 1 << 8, 16, 8, 8)), True), (prompt(shape(1 << 20, 1 << 8, 16, 8, 8)), False)],
    "columns": [(prompt(shape((1 << 18) - 1, 1 << 8, 16, 256, 256)), True), (prompt(shape(1 << 18, 1 << 8, 16, 256, 256)), False)],
    "joins": [(prompt(shape((1 << 20) - 1, 1 << 20, 1, 128, 128)), True), (prompt(shape(1 << 20, 1 << 20, 1, 128, 128)), False)],
    "gradients": [(backward(shape((1 << 19) - 1, 1 << 8, 16, 256, 8)), True), (backward(shape(1 << 19, 1 << 8, 16, 256, 8)), False)],
    "sums": [(backward(shape(1, (1 << 24) - 256, 16, 64, 64, k=16, v=16, q=8)), True), (backward(shape(1, 1 << 25, 16, 64, 128, k=16, v=8, q=16)), False)],
    "steps": [(step(shape((1 << 20) - 1, (1 << 20) - 1, 16, 8, 8)), True), (step(shape(1 << 20, 1 << 20, 16, 8, 8)), False)],
    "lookups": [(lookup((1 << 28) - 16, 512), True), (lookup(1 << 28, 512), False)],
    "few tokens": [(gradient(10, (1 << 29) - 64, 8), True), (gradient(10, 1 << 29, 8), False)],
    "many tokens": [(gradient((1 << 28) - 8192, 1000, 257, 1), False), (gradient(5000, (1 << 30), 8), False), (gradient(5000, (1 << 29), 8), True)],
}


@pytest.mark.parametrize("name", CASES)
def test_grids_that_no_launch_holds(run, name):
    for (rc, kernels), (call, fits) in zip(run([c for c, _ in CASES[name]]), CASES[name]):
        assert all(grid * block < 1 << 32 for _, grid, block in kernels), (call, kernels)
        assert (rc == tcuscan.OK and kernels) if fits else (rc == tcuscan.ERR_UNSUPPORTED and not kernels), (call, rc, kernels)
