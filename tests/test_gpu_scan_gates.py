"""The gated recurrence with closed gates: decays far below 1 and exact limits, against the fp64 recurrence.

Tolerances are those of test_gpu_scan: fields in bf16 2^-8, fp32 fields and states 2e-5 of the norm and
1e-4 of the largest.  They hold at every gate alike: a and 1 - a are both known to a few 2^-24 of
themselves, so every product of them is."""
import numpy as np
import pytest

import _scan_ref as ref
from _util import rel_errors, to_np

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")

BOUND = {"bf16": (2.0 ** -8, 2.0 ** -8), "f32": (2e-5, 1e-4)}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def near(got, want, dtype, what, fp32=None):
    l2, mx = rel_errors(got, want)
    bl, bm = (fp32, fp32) if fp32 and dtype == "f32" else BOUND[dtype]
    assert l2 <= bl and mx <= bm, f"{what}: l2 {l2:.3e} > {bl} or max {mx:.3e} > {bm}"


def check(x, g, dy, leak, dtype, seed=0, fp32=None):
    B, L, D = x.shape
    rng = np.random.default_rng(seed)
    h0, dh = (torch.from_numpy(rng.standard_normal((B, D))).float().cuda() for _ in range(2))
    y, dx, dg = (torch.empty_like(x) for _ in range(3))
    state, dh0 = torch.empty_like(h0), torch.empty_like(h0)
    saved = rlm.scan_saved(B, L, D)
    rlm.rlm_scan_prefill(x, g, y, leak=leak, state_in=h0, state_out=state, saved=saved)
    rlm.rlm_scan_backward(dy, x, g, saved, dx, dg, leak=leak, d_state_out=dh, d_state_in=dh0)
    xs, gs, ds = to_np(x), to_np(g), to_np(dy)
    wy, ws, before = ref.forward(xs, gs, leak, h0.cpu().numpy())
    wx, wg, w0 = ref.backward(ds, xs, gs, leak, before, dh.cpu().numpy())
    near(to_np(y), wy, dtype, "y", fp32)
    near(to_np(state), ws, "f32", "state", fp32)
    near(to_np(dx), wx, dtype, "dx", fp32)
    near(to_np(dg), wg, dtype, "dg", fp32)
    near(to_np(dh0), w0, "f32", "d_state_in", fp32)


def fields(B, L, D, dtype, seed):
    rng = np.random.default_rng(seed)
    x, dy, n = (torch.from_numpy(rng.standard_normal((B, L, D))) for _ in range(3))
    return x.to("cuda", DT[dtype]), dy.to("cuda", DT[dtype]), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("leak", [True, False])
@pytest.mark.parametrize("level", [4.0, 0.0, -4.0, -8.0, -12.0, -16.0, -20.0, -40.0])
def test_gates_about_a_level(level, leak, dtype):
    x, dy, n = fields(3, 300, 72, dtype, 1)
    check(x, (level + 0.25 * n).to("cuda", DT[dtype]), dy, leak, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("leak", [True, False])
@pytest.mark.parametrize("shape", [(2, 500, 64), (1, 4096, 64), (40, 130, 328)])
def test_gates_open_and_closed(shape, leak, dtype):
    """Gates anywhere from -20 to 20."""
    x, dy, n = fields(*shape, dtype, 2)
    check(x, (20 * torch.tanh(n)).to("cuda", DT[dtype]), dy, leak, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("leak", [True, False])
def test_channels_that_hold_one_gate(leak, dtype):
    """Where a gate never changes, the rounding of a decay near 1 is the same at every token and adds up: within
    2^-24 a token, L 2^-24 in fp32."""
    L, D = 4096, 64
    x, dy, _ = fields(1, L, D, dtype, 2)
    g = torch.linspace(-20, 20, D).expand(1, L, D).to("cuda", DT[dtype])
    check(x, g.contiguous(), dy, leak, dtype, fp32=L * 2.0 ** -24)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("leak", [True, False])
@pytest.mark.parametrize("at", [0, 5, 8, 64, 199])
def test_keep_and_forget_are_exact(at, leak, dtype):
    """A state of 1e4 is kept by g = inf to the last bit, and gone after g = -inf."""
    L, D = 200, 16
    x = torch.zeros(1, L, D, dtype=DT[dtype], device="cuda")
    g = torch.full_like(x, float("inf"))
    h0 = torch.full((1, D), 1e4, device="cuda")
    y, state = torch.empty_like(x), torch.empty_like(h0)
    x[:, at], g[:, at] = 2.0 ** -10, float("-inf")
    rlm.rlm_scan_prefill(x, g, y, leak=leak, state_in=h0, state_out=state)
    assert (y[:, :at].float() == h0.to(x.dtype).float()[:, None]).all()
    assert (y[:, at:] == 2.0 ** -10).all() and (state == 2.0 ** -10).all()
    st = h0.clone()
    rlm.rlm_scan_decode(x[:, at], g[:, at], st, y[:, 0], leak=leak)
    assert (st == 2.0 ** -10).all() and (y[:, 0] == 2.0 ** -10).all()
    keep = torch.full_like(g[:, 0], float("inf"))
    st = h0.clone()
    rlm.rlm_scan_decode(torch.zeros_like(x[:, 0]), keep, st, y[:, 0], leak=leak)
    assert torch.equal(st, h0)


@pytest.mark.parametrize("leak", [True, False])
def test_decode_with_closed_gates(leak):
    """One step from a large state: what is left of it is a h, to fp32's last bits."""
    D = 4096
    rng = np.random.default_rng(3)
    g = torch.from_numpy(rng.uniform(-60, 20, (1, D))).float().cuda()
    h = torch.from_numpy(1e4 * rng.standard_normal((1, D))).float().cuda()
    x = torch.from_numpy(1e-3 * rng.standard_normal((1, D))).float().cuda()
    old = to_np(h)
    want, _, _ = ref.forward(to_np(x)[:, None], to_np(g)[:, None], leak, old)
    y = torch.empty_like(x)
    rlm.rlm_scan_decode(x, g, h, y, leak=leak)
    # a and 1 - a are within 2^-21 of themselves (exponential, reciprocal, product); two sums round.
    bound = 2.0 ** -20 * (np.abs(to_np(x)) + ref.sigmoid(to_np(g)) * np.abs(old))
    assert (np.abs(to_np(y) - want[:, 0]) <= bound).all()
