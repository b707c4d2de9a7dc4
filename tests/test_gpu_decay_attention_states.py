"""States are kept as fp32 sums keep them, also where the last tokens of a row add nothing and what is left was added in an earlier segment."""
import numpy as np
import pytest

import attention_reference as ref
from test_gpu_decay_attention import KINDS, Case
from test_gpu_decay_attention_rounding import put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("quiet", [3, 6, 11, 20])
@pytest.mark.parametrize("lengths", [[323], [326, 64, 331], [1290]], ids=str)
def test_states_after_tokens_that_add_nothing(kind, quiet, lengths):
    """Rows whose last `quiet` keys, and first `quiet` queries, are zeros; segments are 64 tokens."""
    c = Case(kind, lengths, heads=(2, 2, 2), dk=32, dv=32, decays=[0.5, 0.6], seed=71)
    q, k = c.host[0].copy(), c.host[1].copy()
    for lo, hi in zip(c.offsets, c.offsets[1:]):
        q[lo:lo + quiet] = 0.0
        k[hi - quiet:hi] = 0.0
    zero = np.zeros((c.rows, 2, 32, 32))
    put(c, q=q, k=k, s0=zero, ds=zero)
    args = (*c.host, c.g.double().numpy(), c.offsets, c.scale, c.s0.numpy())
    pairs = [(c.forward()[1], ref.forward(*args)[1]), (c.backward()[3], ref.backward(*args, c.do.double().numpy(), c.ds.numpy())[3])]
    for got, want in pairs:
        off = got.double().cpu().numpy() - want
        for r in range(c.rows):
            for h in range(2):
                # sixteen roundings to 24 bits, all to the same side; values in two bf16 parts would be off by up to 2^-16 each
                assert np.linalg.norm(off[r, h]) <= 2.0 ** -20 * np.linalg.norm(want[r, h])
