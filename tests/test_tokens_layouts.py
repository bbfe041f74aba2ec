"""CPU tests: which layouts the C entries of the operators among a request's tokens refuse because an output would write what
another tensor, or another of its own heads, holds (pointers below are never followed: every call is refused)."""
import pytest

from paper_2107_06960_amd import mafat as M
from test_tokens_abi import A, B, C, D, E, F, _decay, _rotary

WIDTH = 64 * 2  # bytes of a head
ROW = 4 * 3 * 64  # elements of a row of four heads of queries, keys and values
BY_HEAD = dict(rows=8, q_heads=4, k_heads=4, q_row=ROW, q_head=192, k_row=ROW, k_head=192, qy_row=ROW, qy_head=192, ky_row=ROW, ky_head=192)


@pytest.mark.parametrize("shape, call", [
    # keys half a head into the queries; in the next head's queries; a row further down; and half of one there
    (BY_HEAD, dict(q=C, qy=C, k=C + WIDTH // 2, ky=C + WIDTH // 2)), (BY_HEAD, dict(q=C, qy=C, k=C + 3 * WIDTH, ky=C + 3 * WIDTH)),
    (BY_HEAD, dict(q=C, qy=C, k=C + 7 * 2 * ROW, ky=C + 7 * 2 * ROW)),
    (BY_HEAD, dict(q=C + 7 * 2 * ROW + 2 * WIDTH + WIDTH // 2, qy=C + 7 * 2 * ROW + 2 * WIDTH + WIDTH // 2, k=C, ky=C)),
    # heads outside of rows
    (dict(BY_HEAD, q_row=64, qy_row=64, k_row=64, ky_row=64, q_head=64 * 16, qy_head=64 * 16, k_head=64 * 16, ky_head=64 * 16),
     dict(q=C, qy=C, k=C + WIDTH * 7, ky=C + WIDTH * 7)),
    # other strides
    (dict(BY_HEAD, k_head=128, ky_head=128), dict(q=C, qy=C, k=C + WIDTH, ky=C + WIDTH)),
])
def test_rotary_refuses_keys_in_the_queries_way(shape, call):
    assert _rotary(shape, call) == M.MAFAT_EINVAL and b"overlaps another tensor" in M.lib().mafat_last_error()


@pytest.mark.parametrize("shape, call", [
    # rows of two heads a head apart; rows half a head into the next ones; three heads up are two rows down
    (dict(qy_row=64, qy_head=64), {}), (dict(ky_row=96, ky_head=64), {}), (dict(qy_row=192, qy_head=128), {}),
    (dict(q_row=64, qy_row=64, q_head=64, qy_head=64), dict(qy=C)),
])
def test_rotary_refuses_outputs_in_their_own_way(shape, call):
    assert _rotary(shape, call) == M.MAFAT_EINVAL and b"overlap each other" in M.lib().mafat_last_error()


@pytest.mark.parametrize("shape, call, why", [
    (dict(y_row=32, y_head=32), {}, b"overlap each other"), (dict(y_row=96, y_head=64), {}, b"overlap each other"),
    # y between the queries' heads, and half a head off
    (dict(q_row=4 * 96, q_head=96, y_row=4 * 96, y_head=96), dict(y=A + 2 * 48), b"overlaps an input"),
    (dict(v_row=128, v_head=64, y_row=128, y_head=64, q_heads=2), dict(y=C + 2 * 64), b"overlaps an input"),
])
def test_decay_attention_refuses_outputs_in_the_way(shape, call, why):
    assert _decay(shape, call) == M.MAFAT_EINVAL and why in M.lib().mafat_last_error()
