"""What the gated recurrence's entry points refuse, each for its own reason (no GPU: nothing is enqueued).
Calls have no launch context, so one that is not refused says so."""
import pytest

import paper_2607_05583_gb300 as rlm
from test_scan_cpu import FAKE, GB, backward, field, lib  # noqa: F401

BACKWARD = [(dict(saved=None), b"saved is NULL"), (dict(dx=field(1)), b"dx or dg overlaps"),
            (dict(dg=field(3)), b"dx and dg overlap"), (dict(dy=field(0, B=3)), b"dy must have x's shape"),
            (dict(dsin=FAKE + 12 * GB), b"d_state_in overlaps saved"),
            (dict(dg=field(4, dt=rlm.RLM_F32)), b"dg must have x's shape and dtype"),
            (dict(dx=field(3, sl=0, sb=0)), b"dx has overlapping rows"), (dict(x=field(1, off=8)), b"16-byte aligned"),
            (dict(saved=FAKE + 12 * GB + 4), b"saved is not 16-byte aligned"),
            (dict(saved=FAKE + 3 * GB), b"saved overlaps a field"), (dict(dsin=FAKE + 2 * GB), b"d_state_in overlaps a field"),
            (dict(dg=field(4, sb=64)), b"dg has overlapping rows"), (dict(g=None, dy=field(2, L=99)), b"dy must have")]


@pytest.mark.parametrize("k", range(len(BACKWARD)))
def test_backward_refusals_have_their_reasons(lib, k):  # noqa: F811
    kw, why = BACKWARD[k]
    assert backward(lib, **kw) == rlm.RLM_ERR_INVALID_ARG
    assert why in lib.rlm_last_error(), (kw.keys(), lib.rlm_last_error())
