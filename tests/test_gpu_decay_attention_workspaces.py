"""Calls in the workspace of a larger call, which holds other segments at other places or none."""
import pytest

from test_gpu_decay_attention import Case
from paper_2411_17887_amd import tcuscan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,larger", [([512], (2, 512)), ([300], (2, 512)), ([4096], (1, 4352)), ([700, 1300], (5, 9000))], ids=str)
def test_calls_in_the_workspace_of_a_larger_one(kind, lengths, larger):
    c = Case(kind, lengths, heads=(8, 8, 8), dk=64, dv=64, seed=42)
    ws = tcuscan.new_decay_attention_workspace(*larger, 8, 64, 64, dt=kind)
    c.check_forward(*c.forward(ws))
    ws[32:] = -1                                               # NaN
    c.check_forward(*c.forward(ws))
    ws = tcuscan.new_decay_attention_backward_workspace(*larger, 8, 64, 64, dt=kind)
    ws[32:] = -1
    c.check_backward(*c.backward(ws))
