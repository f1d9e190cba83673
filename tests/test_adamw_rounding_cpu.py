"""Argument checks of the 8-bit moments' rounding (no GPU: nothing is enqueued)."""
import paper_2607_05583_gb300 as rlm
from test_adamw_cpu import SCALES, call, entry, lib  # noqa: F401


def test_roundings_of_8_bit_moments(lib):  # noqa: F811
    draw = rlm.ADAMW_DRAW
    for bits in (8, 8 | draw):
        assert call(lib, [entry(**SCALES)], bits=bits) == rlm.RLM_ERR_INVALID_ARG
        assert b"launch is NULL" in lib.rlm_last_error()
        assert call(lib, [entry()], bits=bits) == rlm.RLM_ERR_INVALID_ARG and b"scales" in lib.rlm_last_error()
    for bits in (32 | draw, draw, 8 | 2 * draw):
        assert call(lib, [entry(**SCALES)], bits=bits) == rlm.RLM_ERR_INVALID_ARG and b"bits=" in lib.rlm_last_error()
