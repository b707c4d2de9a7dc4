"""A decay that is not a number makes everything of its head so, and nothing of other heads."""
import pytest

from test_gpu_decay_attention import KINDS, Case
from paper_2411_17887_amd import tcuscan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths", [[50, 1], [700, 40]], ids=str)
def test_decays_that_are_not_a_number(kind, lengths):
    import torch
    c = Case(kind, lengths, heads=(3, 3, 3), dk=32, dv=48, seed=43)
    want = [*c.forward(), *c.backward()]
    c.log_decay[1] = float("nan")
    got = [*c.forward(), *c.backward()]
    for w, g in zip(want, got):
        assert torch.equal(g[:, 0], w[:, 0]) and torch.equal(g[:, 2], w[:, 2]) and torch.isnan(g[:, 1]).all()


@pytest.mark.parametrize("kind", KINDS)
def test_decays_that_are_not_a_number_in_single_tokens(kind):
    import torch
    c = Case(kind, [1] * 5, heads=(2, 2, 2), dk=32, dv=48, seed=44)
    c.log_decay[0] = float("nan")
    out, state = torch.zeros(5, 2, 48, dtype=c.dt, device="cuda"), c.s0.cuda()
    tcuscan.decay_attention_step(*c.qkv, out, c.log_decay, state, scale=c.scale)
    torch.cuda.synchronize()
    assert torch.isnan(out[:, 0]).all() and torch.isnan(state[:, 0]).all()
    assert torch.isfinite(out[:, 1]).all() and torch.isfinite(state[:, 1]).all()
