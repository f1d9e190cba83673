"""One row has no pitch: a residual that is y itself is taken whatever their row pitches say (no GPU)."""
import paper_2607_05583_gb300 as rlm
from test_linear_cpu import FAKE, GB, K, N, forward, lib, mat  # noqa: F401


def test_a_residual_in_place_of_one_row(lib):  # noqa: F811
    one = dict(x=mat(0, 1, K), y=mat(4, 1, N, ld=N), pre=None)
    for residual in (mat(4, 1, N, ld=N), mat(4, 1, N, ld=4 * N)):
        assert forward(lib, residual=residual, **one) == rlm.RLM_ERR_INVALID_ARG
        assert b"launch is NULL" in lib.rlm_last_error(), lib.rlm_last_error()
    assert forward(lib, residual=mat(4, 1, N, off=16), **one) == rlm.RLM_ERR_INVALID_ARG
    assert b"residual overlaps" in lib.rlm_last_error()
