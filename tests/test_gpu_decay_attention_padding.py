"""Tokens in front of the first row and behind the last one, in gradients that are put together from several heads: such tokens are neither read nor
written, whatever the workspace holds from calls before."""
import pytest

from test_gpu_decay_attention import KINDS, Case
from paper_2411_17887_amd import tcuscan

pytestmark = pytest.mark.gpu


# four elements a thread | one; cut into segments or not; rows that leave no token at all to the call
@pytest.mark.parametrize("dk,dv,packed", [(64, 32, False), (13, 6, False), (12, 20, True)])
@pytest.mark.parametrize("lengths", [[100, 0, 67], [900, 30], [0]], ids=str)
@pytest.mark.parametrize("heads", [(4, 1, 1), (1, 4, 2), (2, 2, 4)], ids=str)
@pytest.mark.parametrize("kind", KINDS)
def test_gradients_of_shared_heads_leave_tokens_of_no_row_alone(kind, heads, lengths, dk, dv, packed):
    c = Case(kind, lengths, heads=heads, all_heads=4, dk=dk, dv=dv, gap=5, packed=packed, seed=41)
    ws = tcuscan.new_decay_attention_backward_workspace(c.rows, c.total, 4, dk, dv, *heads, dt=kind)
    ws[32:] = -1                                               # NaN everywhere but in the header
    c.check_backward(*c.backward(ws))                          # (which looks at the guards in front and behind, too)
