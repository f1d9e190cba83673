"""The selective scan's long memory: states that overflow, states that stay zero under growing decays, steps of which only some
are open, and lengths and widths about the kernels' tiles and blocks."""
import math

import pytest

import _ssm_ref as ref
from test_gpu_ssm import check, gen, inputs

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


# Which of a sequence's tokens move the states (place in 32, steps about).
PATTERNS = {"all": (lambda t: t >= 0, 0.005), "only the 16th": (lambda t: t % 32 == 16, 0.005), "only the 15th": (lambda t: t % 32 == 15, 0.005),
            "all but the 16th": (lambda t: t % 32 != 16, 0.005), "all but the 15th": (lambda t: t % 32 != 15, 0.005),
            "only the first of 64": (lambda t: t % 64 == 0, 0.005), "every other 16": (lambda t: t // 16 % 2 == 0, 0.005),
            "0 to 0.02": (None, 0.01), "all, slowly": (lambda t: t >= 0, 0.0003), "all, fast": (lambda t: t >= 0, 0.05)}


@pytest.mark.parametrize("N,rows", [(8, 1), (8, 300), (32, 1), (32, 76)])
def test_steps_that_depend_on_their_place(N, rows):
    """States and gradients that only grow, with most of the steps 0 or not: the mean errors of the final state, of the initial
    state's gradient and of dA, per pattern.  One row runs in segments; with enough empty rows beside it a block walks all of it.

    Over a tile (16 tokens) that moves the states at all, what is carried takes e^(A sum of D), off in the mean by 8e-9 of itself
    at most; a state remembers 1 / E such tiles, E the mean of what they forget, and no more than there are.  What enters is off
    once by the exponentials' means (3.1e-8 each at most) over the tokens between corrections, 32.  Single roundings (three of
    at most 2^-24 a token) cancel over a pattern's channels and states but for their root."""
    B, L, per = 1, 8192, 24
    g = gen(N)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    t = torch.arange(L, device="cuda")
    D = per * len(PATTERNS)
    dt = torch.empty(B, L, D, device="cuda")
    for k, (fn, step) in enumerate(PATTERNS.values()):
        r = rand(B, L, per)
        dt[..., k * per:(k + 1) * per] = 0.02 * r if fn is None else step * (0.8 + 0.4 * r) * fn(t)[None, :, None]
    x, b, c, dy = 0.5 + rand(B, L, D), 0.5 + rand(B, L, N), 0.5 + rand(B, L, N), 0.5 + rand(B, L, D)
    A, dh = -torch.ones(D, N, device="cuda"), 0.5 + rand(B, D, N)
    par = rlm.SsmParams(A, softplus=False)
    lengths = torch.zeros(rows, dtype=torch.int32, device="cuda")
    lengths[0] = L
    ix, idt, ib, ic, idy = (v.expand(rows, -1, -1) for v in (x, dt, b, c, dy))
    y, state, saved = torch.empty(rows, L, D, device="cuda"), torch.empty(rows, D, N, device="cuda"), rlm.ssm_saved(rows, L, D, N)
    assert (rlm.rlm_ssm_workspace_size(rows, L, D, N) == 0) == (rows > 1)
    rlm.rlm_ssm_prefill(ix, idt, ib, ic, par, y, state_out=state, saved=saved, lengths=lengths)
    out = [torch.empty_like(y) for _ in range(2)] + [torch.empty(rows, L, N, device="cuda") for _ in range(2)]
    dh0, gr = torch.empty_like(state), rlm.SsmGrads.empty(D, N)
    rlm.rlm_ssm_backward(idy, ix, idt, ib, ic, par, saved, *out, gr, d_state_out=dh.expand(rows, -1, -1).contiguous(), d_state_in=dh0,
                         lengths=lengths)
    h, before = torch.zeros(B, D, N, dtype=torch.float64, device="cuda"), torch.empty(L, B, D, N, dtype=torch.float64, device="cuda")
    for i in range(L):
        before[i] = h
        d = dt[:, i, :, None].double()
        h = torch.exp(-d) * h + d * x[:, i, :, None].double() * b[:, i, None, :].double()
    G, dA = dh.double(), torch.zeros(D, N, dtype=torch.float64, device="cuda")
    for i in range(L - 1, -1, -1):
        d = dt[:, i, :, None].double()
        G = torch.exp(-d) * (G + dy[:, i, :, None].double() * c[:, i, None, :].double())
        dA += (G * d * before[i]).sum(0)
    far = []
    for k, name in enumerate(PATTERNS):
        at = slice(k * per, (k + 1) * per)
        tiles = dt[..., at].double().view(B, L // 16, 16, per).sum(2)
        live = (tiles > 0).double().mean().item() * (L // 16)
        forget = tiles.sum(1).mean().item() / live               # of a tile that moves the states
        n = min(1 / -math.expm1(-forget), live)                 # tiles remembered
        tokens = n * (dt[..., at] > 0).sum().item() / per / live
        one = 8e-9 * n + 32 * 3.1e-8 + 9 * 2.0 ** -24 * math.sqrt(tokens / (per * N))
        for what, got, want, bound in (("state", state[:1, at], h[:, at], one), ("dh0", dh0[:1, at], G[:, at], one), ("dA", gr.A[at], dA[at], 2 * one)):
            e = (got / want - 1).mean().item()
            if not abs(e) <= bound:
                far.append((name, what, e, bound))
    assert not far, far


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [8, 16, 32])
@pytest.mark.parametrize("L,D", [(8, 56), (9, 64), (15, 72), (16, 64), (17, 120), (31, 128), (32, 136), (33, 56), (47, 256), (48, 264), (49, 128)])
def test_lengths_and_widths_about_tiles_and_blocks(L, D, N, dtype):
    """Tiles are of 16 tokens (of 8 in the forward pass at N = 8), states are put right every 32, a forward block has 1024 / N
    channels and a gradient's 64."""
    check(inputs(2, L, D, N, dtype, gen(L), view=L % 2 == 1), gate=L % 3 != 0)
