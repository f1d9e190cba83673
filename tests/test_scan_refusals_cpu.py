"""What the gated recurrence's entry points refuse, each for its own reason, and views that they take (no GPU:
nothing is enqueued).  Calls have no launch context, so one that is not refused says so."""
import pytest

import paper_2607_05583_gb300 as rlm
from test_scan_cpu import FAKE, GB, backward, ctypes, field, lib, prefill  # noqa: F401

NO_LAUNCH = ctypes.POINTER(rlm._Launch)()

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


def reaches_the_launch(status, lib):  # noqa: F811
    return status == rlm.RLM_ERR_INVALID_ARG and b"launch is NULL" in lib.rlm_last_error()


# (stride_b, stride_l) of [2][100][64] halves of one buffer of twice the width: batch rows first, time first, and
# rows with room between them.
@pytest.mark.parametrize("sb,sl", [(12800, 128), (128, 256), (128, 512), (25600, 256), (20000, 160)])
def test_halves_of_one_buffer_are_apart(lib, sb, sl):  # noqa: F811
    half = lambda k, off: field(k, sb=sb, sl=sl, off=off)
    assert reaches_the_launch(backward(lib, dx=half(3, 0), dg=half(3, 128)), lib), lib.rlm_last_error()
    assert reaches_the_launch(backward(lib, dx=half(3, 128), dg=half(3, 0)), lib), lib.rlm_last_error()
    assert reaches_the_launch(prefill(lib, x=half(0, 0), y=half(0, 128), ln=NO_LAUNCH), lib), lib.rlm_last_error()
    assert backward(lib, dx=half(3, 0), dg=half(3, 112)) == rlm.RLM_ERR_INVALID_ARG
    assert b"dx and dg overlap" in lib.rlm_last_error()
    assert prefill(lib, x=half(0, 0), y=half(0, 2 * sb), ln=NO_LAUNCH) == rlm.RLM_ERR_INVALID_ARG    # the next batch row
    assert b"y overlaps" in lib.rlm_last_error()
