"""How much of the sum of the terms' sizes the kernels may round before the output's own rounding, on inputs whose terms cancel: what rounds scores, states or what
is added to states to fewer bits than the header says is far outside.

An operand in two bf16 parts is off by 2^-16 of itself, in three by 2^-24.  bf16 inputs are one part, f16 inputs two and exact.  So, in units of the terms:
  bf16  added to a state 2^-16, the state read 2^-16 (scores: 2^-16)
  f16   the same, and two products of low parts left out, 2^-16 each
  f32   four products of operands in three parts on a path, of each what lies below the third part and two products of 2^-24
and 2^-21 for the weights a^n (x e^-x <= 1/2 of their exponents' rounding), 2^-24 for every addition of a chain of fp32 sums."""
import numpy as np
import pytest

import attention_reference as ref
from test_gpu_decay_attention import KINDS, Case

pytestmark = pytest.mark.gpu

INSIDE = {"bf16": 2.0 ** -15, "f16": 2.0 ** -14, "f32": 2.0 ** -21}


def check(got, want, size, kind, longest, features, state=False):
    inside = (INSIDE["f32"] if state else INSIDE[kind]) + 2.0 ** -21 + (features + 64 + longest / 16) * 2.0 ** -24
    bound = ref.UNIT["f32" if state else kind] * np.abs(want) + inside * size + 1e-30
    if kind == "f16" and not state:
        bound = bound + 2.0 ** -25
    there = ~np.isnan(want)
    off = (np.abs(got.double().cpu().numpy() - want) / bound)[there]
    assert (off <= 1.0).all(), f"{off.max():.3g} of what rounding explains"


def check_all(c):
    args = (*c.host, c.g.double().numpy(), c.offsets, c.scale, c.s0.numpy())
    for i, (got, want, size) in enumerate(zip(c.forward(), ref.forward(*args), ref.forward(*args, absolute=True))):
        check(got, want, size, c.kind, c.longest, c.features, state=i == 1)
    args = (*args, c.do.double().numpy(), c.ds.numpy())
    for i, (got, want, size) in enumerate(zip(c.backward(), ref.backward(*args), ref.backward(*args, absolute=True))):
        check(got, want, size, c.kind, c.longest, c.features, state=i == 3)


def put(c, q=None, k=None, v=None, do=None, s0=None, ds=None):
    """Other inputs in the place of the case's."""
    import torch
    for i, x in enumerate((q, k, v)):
        if x is not None:
            x = torch.from_numpy(x).to(c.dt)
            c.host[i], c.qkv[i] = x.double().numpy(), x.cuda()
    if do is not None:
        c.do = torch.from_numpy(do).to(c.dt)
    if s0 is not None:
        c.s0 = torch.from_numpy(s0).float()
    if ds is not None:
        c.ds = torch.from_numpy(ds).float()


def alternating(n, heads, features, a, rng, from_end=False):
    """Values of six bits, every second one minus a (a multiple of 1/4) times the one before it: behind a decay of `a` they cancel."""
    x = rng.randint(32, 64, (n, heads, features)) / 64.0 * rng.choice((-1.0, 1.0), (n, heads, features))
    x = x[::-1] if from_end else x
    x[1::2] = -a * x[: n - n % 2: 2]
    return np.ascontiguousarray(x[::-1] if from_end else x)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths", [[31], [9, 64, 20], [700]], ids=str)
@pytest.mark.parametrize("which", ["o", "dq", "dk", "dv"])
def test_scores_whose_terms_cancel(kind, lengths, which):
    """Scores of one sign, values that cancel in pairs: what is rounded of a score is not rounded alike in the next one."""
    c = Case(kind, lengths, heads=(2, 2, 2), dk=32, dv=32, decays=[0.75, 0.75], seed=51)
    rng = np.random.RandomState(52)
    n = c.total

    def ones():
        x = rng.uniform(0.5, 1.0, (n, 2, 32))
        x[1::2] = x[: n - n % 2: 2]                            # (keys come in pairs, too)
        return x

    zero = np.zeros((c.rows, 2, 32, 32))
    pairs = alternating(n, 2, 32, 0.75, rng, from_end=which in ("dk", "dv"))
    put(c, **{"o": dict(q=ones(), k=ones(), v=pairs), "dq": dict(do=ones(), v=ones(), k=pairs), "dv": dict(k=ones(), q=ones(), do=pairs),
              "dk": dict(v=ones(), do=ones(), q=pairs)}[which], s0=zero, ds=zero)
    check_all(c)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("decay", [1.0, 0.9])
@pytest.mark.parametrize("lengths", [[20], [70, 300]], ids=str)
def test_states_whose_terms_cancel_where_they_are_read(kind, decay, lengths):
    """Rows of a state that are minus 3/4 of the row before, read by (3/4, 1, 3/4, 1, ...)."""
    c = Case(kind, lengths, heads=(2, 2, 2), dk=32, dv=32, decays=[decay] * 2, seed=53)
    rng = np.random.RandomState(54)
    reader = np.tile([0.75, 1.0], 16)
    s0 = rng.randint(1 << 21, 1 << 22, (c.rows, 2, 32, 32)) / float(1 << 16) * rng.choice((-1.0, 1.0), (c.rows, 2, 32, 32))
    s0[..., 1::2, :] = -0.75 * s0[..., ::2, :]
    every = np.broadcast_to(reader, (c.total, 2, 32)).copy()
    put(c, q=every, s0=s0)                                     # o = q S
    check_all(c)
    put(c, k=every, ds=s0)                                     # dv = k R
    check_all(c)
    turned = np.ascontiguousarray(s0.swapaxes(-1, -2))
    put(c, do=every, s0=turned)                                # dq = do S^T
    check_all(c)
    put(c, v=every, ds=turned)                                 # dk = v R^T
    check_all(c)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths", [[45], [64, 500]], ids=str)
@pytest.mark.parametrize("which", ["o", "dq", "dk", "dv"])
def test_tokens_that_cancel_in_a_state(kind, lengths, which):
    """Tokens in pairs of opposite contributions whose weighted values have different bits, read from the state by later tokens."""
    decay = 0.9
    c = Case(kind, lengths, heads=(2, 2, 2), dk=32, dv=32, decays=[decay] * 2, seed=55)
    rng = np.random.RandomState(56)
    n = c.total
    from_end = which in ("dk", "dv")
    values = rng.uniform(0.5, 1.0, (n, 2, 32))
    keys = rng.uniform(0.5, 1.0, (n, 2, 32))
    if from_end:
        values, keys = values[::-1], keys[::-1]
    even = slice(0, n - n % 2, 2)
    values[1::2] = 0.75 * decay * values[even]
    keys[1::2] = -keys[even] / 0.75
    if from_end:
        values, keys = values[::-1], keys[::-1]
    values, keys, readers = np.ascontiguousarray(values), np.ascontiguousarray(keys), rng.uniform(0.5, 1.0, (n, 2, 32))
    zero = np.zeros((c.rows, 2, 32, 32))
    put(c, **{"o": dict(q=readers, k=keys, v=values), "dq": dict(do=readers, v=keys, k=values), "dv": dict(k=readers, q=keys, do=values),
              "dk": dict(v=readers, do=keys, q=values)}[which], s0=zero, ds=zero)
    check_all(c)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths,dk,dv", [([1, 0, 33, 200], 64, 64), ([1500], 128, 96), ([300, 40], 20, 70), ([90], 256, 256)], ids=str)
def test_inputs_at_random(kind, lengths, dk, dv):
    check_all(Case(kind, lengths, heads=(2, 2, 2), dk=dk, dv=dv, seed=57))


@pytest.mark.parametrize("kind", KINDS)
def test_shared_heads(kind):
    check_all(Case(kind, [150, 20], heads=(4, 2, 1), dk=48, dv=32, seed=58))
