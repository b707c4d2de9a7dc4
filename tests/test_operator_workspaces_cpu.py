"""One workspace for calls of different sizes: what is allocated for the largest holds all smaller ones (no GPU; addresses are never followed)."""
import random

import pytest

import launch_recorder
from operator_launches import launches, shape
from paper_2411_17887_amd import tcuscan

AT = [0x100000 * (i + 1) for i in range(12)]
KINDS = [(8, 64, 64), (16, 128, 128), (1, 128, 128), (4, 32, 48), (12, 256, 96), (300, 16, 16), (700, 8, 8)]


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    shim = launch_recorder.build(tmp_path_factory.mktemp("shim"))
    return lambda calls: launches(shim, calls)


def prompt(rows, total, heads, dk, dv, ws_bytes):
    return ("tcuscan_decay_attention", [shape(rows, total, heads, dk, dv), *AT[:6], tcuscan.BF16_F32, AT[6], AT[7], 0, rows, AT[8], ws_bytes, 0])


def backward(rows, total, heads, dk, dv, ws_bytes, k=0):
    return ("tcuscan_decay_attention_backward", [shape(rows, total, heads, dk, dv, k=k), *AT[:9], tcuscan.F16_F32, AT[9], 0, 0, AT[10], ws_bytes, 0])


def sizes(heads, dk, dv, seed):
    """Pairs of rows and tokens, on both sides of where segments change their lengths, and at random."""
    rng = random.Random(seed)
    edges = [t + d for t in (256, 512, *(2 ** i // g for i in range(13, 24) for g in (1, heads))) for d in (-1, 0, 1) if 0 < t + d < 1 << 20]
    return [(rng.choice((1, 1, 2, 3, 17)), t) for t in edges] + [(rng.randint(1, 60), int(2 ** rng.uniform(0, 19))) for _ in range(60)]


@pytest.mark.parametrize("heads,dk,dv", KINDS)
@pytest.mark.parametrize("grads", [False, True])
def test_a_workspace_serves_all_smaller_calls(run, heads, dk, dv, grads):
    some = sizes(heads, dk, dv, 1)
    shared = heads // 4 if heads % 4 == 0 else 0

    def need(rows, total):
        return tcuscan.decay_attention_workspace_bytes(rows, total, heads, dk, dv, k_heads=shared if grads else None, backward=grads)

    rng = random.Random(2)
    pairs = []
    for rows, total in some:
        smaller = [s for s in some if s[0] <= rows and s[1] <= total]
        pairs += [(need(rows, total), s) for s in rng.sample(smaller, min(12, len(smaller)))]
    for (rc, kernels), (have, (rows, total)) in zip(run([backward(*s, heads, dk, dv, have, shared) if grads else prompt(*s, heads, dk, dv, have) for have, s in pairs]), pairs):
        assert rc == tcuscan.OK and kernels, (have, rows, total)
    # and beyond the calls that may or may not be cut, what is asked for grows
    some = sorted(s for s in some if s[1] > 512)
    for (r0, t0), (r1, t1) in zip(some, some[1:]):
        assert need(max(r0, r1), max(t0, t1)) >= max(need(r0, t0), need(r1, t1))


def test_short_calls_take_the_workspace_they_get(run):
    """512 tokens are cut in one row and not in two; with the workspace for two rows, one row is not cut either."""
    two, one = (tcuscan.decay_attention_workspace_bytes(r, 512, 8, 64, 64) for r in (2, 1))
    assert two < one
    got = run([prompt(2, 512, 8, 64, 64, two), prompt(1, 512, 8, 64, 64, two), prompt(1, 512, 8, 64, 64, one), prompt(1, 512, 8, 64, 64, two - 1)])
    assert [rc for rc, _ in got] == [tcuscan.OK] * 3 + [tcuscan.ERR_WORKSPACE]
    assert [len(kernels) for _, kernels in got] == [1, 1, 3, 0]


def test_longer_calls_are_refused_a_workspace_that_is_too_small(run):
    for total in (513, 4096, 4352, 65536):
        need = tcuscan.decay_attention_workspace_bytes(1, total, 16, 128, 128)
        (rc, kernels), (least, _) = run([prompt(1, total, 16, 128, 128, 256), prompt(1, total, 16, 128, 128, need)])
        assert rc == tcuscan.ERR_WORKSPACE and not kernels and least == tcuscan.OK
