"""CPU tests: calls of linear attention whose segments pass 31 bits are refused (no pointer below is followed)."""
import pytest

from paper_2107_06960_amd import mafat as M
from paper_2107_06960_amd import operators as O
from test_tokens_abi import CALL, DECAY, _decay

MOST = (1 << 31) - 1
TINY = dict(q_heads=1, kv_heads=1, key_dim=1, value_dim=1, q_row=1, q_head=1, k_row=1, k_head=1, v_row=1, v_head=1, y_row=1, y_head=1,
            decay_row=1, state_slot=1, slots=0)


@pytest.mark.parametrize("rows, requests", [(MOST, MOST - 1), (MOST, MOST - (1 << 23))])
def test_too_many_segments(rows, requests):
    """rows / 128 + requests of them."""
    shape = dict(TINY, rows=rows, requests=requests, dtype=M.MAFAT_BF16, value_dim=8, v_row=8, v_head=8, y_row=8, y_head=8, key_dim=8,
                 q_row=8, q_head=8, k_row=8, k_head=8)
    assert _decay(shape, dict(states=None, slots=None, ws_bytes=1 << 62)) == M.MAFAT_EUNSUPPORTED, M.lib().mafat_last_error()
    with pytest.raises(M.MafatError, match="2\\^31"):
        O.mafat_decay_workspace(O.mafat_decay(**dict(DECAY, **shape)))


def test_as_many_as_fit():
    shape = dict(DECAY, **dict(TINY, rows=MOST, requests=1))
    assert O.mafat_decay_workspace(O.mafat_decay(**shape)) > 0
    # token after token there are no segments
    assert O.mafat_decay_workspace(O.mafat_decay(**dict(shape, requests=MOST))) == 0
    assert CALL["workspace"]
