"""The selective scan's long memory: states that overflow, states that stay zero under growing decays."""
import math

import pytest

import _ssm_ref as ref
from test_gpu_ssm import gen

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")


@pytest.mark.parametrize("N", [8, 16, 32])
@pytest.mark.parametrize("L", [40, 400])
def test_infinite_states_stay(L, N):
    """A state past fp32's range, given or grown, is infinite at the end of a sequence as after single steps; so is the
    gradient of the initial state where the final one's is.  L = 400 runs in segments, L = 40 of 2 tiles too."""
    B, D = 1, 8
    inf = math.inf
    one = lambda *s: torch.ones(*s, device="cuda")  # noqa: E731
    A = torch.zeros(D, N, device="cuda")
    A[1], A[2] = -1e-4, 1.0             # keeps, decays slowly, grows by e a token; channel 3 keeps too
    h0 = one(B, D, N)
    h0[:, 0], h0[:, 1], h0[:, 2], h0[:, 3] = inf, -inf, 1e30, 3e38
    x, b, dt = one(B, L, D), one(B, L, N), one(B, L, D)
    x[..., 3] = 1e36                    # 3e38 + t 1e36 passes the largest fp32 value after 40 tokens
    par = rlm.SsmParams(A, softplus=False)
    y, state, saved = torch.empty_like(x), torch.empty_like(h0), rlm.ssm_saved(B, L, D, N)
    rlm.rlm_ssm_prefill(x, dt, b, b, par, y, state_in=h0, state_out=state, saved=saved)
    step, yt = h0.clone(), torch.empty_like(y)
    for t in range(L):
        rlm.rlm_ssm_decode(x[:, t], dt[:, t], b[:, t], b[:, t], par, step, yt[:, t])
    assert not step.isnan().any()
    where = [0, 1, 2] + [3] * (L > 41)          # (at 40 tokens the last one is at the range's end: either side of it)
    assert step[:, where].isinf().all()
    assert torch.equal(state[:, where], step[:, where]) and torch.equal(y[..., :3].isinf(), yt[..., :3].isinf())
    assert not state.isnan().any()
    dh = one(B, D, N)
    dh[:, 0], dh[:, 1], dh[:, 2] = inf, -inf, 3e38
    out = [torch.empty_like(x) for _ in range(2)] + [torch.empty_like(b) for _ in range(2)]
    dh0, gr = torch.empty_like(h0), rlm.SsmGrads.empty(D, N)
    rlm.rlm_ssm_backward(one(B, L, D), x, dt, b, b, par, saved, *out, gr, d_state_out=dh, d_state_in=dh0)
    assert (dh0[:, 0] == inf).all() and (dh0[:, 1] == -inf).all() and (dh0[:, 2] == inf).all()
    assert dh0[:, 3:].isfinite().all()


@pytest.mark.parametrize("N", [8, 16, 32])
@pytest.mark.parametrize("L", [60, 700])
def test_zero_states_under_growing_decays(L, N):
    """A state that nothing has driven is 0 whatever its decays would make of another, e^(10 t) here; the same for the gradient
    behind the last token that counts.  What the driven end of the sequence leaves is the recurrence's."""
    B, D, n = 1, 8, 5
    g = gen(L)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, dt, b, c, dy = rn(B, L, D), torch.full((B, L, D), 10.0, device="cuda"), rn(B, L, N), rn(B, L, N), rn(B, L, D)
    x[:, :-n], dy[:, n:] = 0, 0
    A = torch.ones(D, N, device="cuda")
    par = rlm.SsmParams(A, softplus=False)
    y, state, saved = torch.empty_like(x), torch.empty(B, D, N, device="cuda"), rlm.ssm_saved(B, L, D, N)
    rlm.rlm_ssm_prefill(x, dt, b, c, par, y, state_out=state, saved=saved)
    end = slice(L - n, L)
    want = ref.ssm(x[:, end], dt[:, end], b[:, end], c[:, end], A, softplus=False)
    ref.assert_within(state, want["state"], "state")
    ref.assert_within(y[:, end], want["y"], "y")
    assert not y[:, :-n].any()
    out = [torch.empty_like(x) for _ in range(2)] + [torch.empty_like(b) for _ in range(2)]
    dh0, gr = torch.empty(B, D, N, device="cuda"), rlm.SsmGrads.empty(D, N)
    rlm.rlm_ssm_backward(dy, x, dt, b, c, par, saved, *out, gr, d_state_in=dh0)
    start = slice(0, n)
    want = ref.ssm(x[:, start], dt[:, start], b[:, start], c[:, start], A, softplus=False, dy=dy[:, start])
    ref.assert_within(dh0, want["dh0"], "dh0")
    ref.assert_within(out[0][:, start], want["dx"], "dx")
    for t in out[:3]:
        assert not t[:, n:].any()
