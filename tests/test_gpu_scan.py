"""The gated linear recurrence on the GPU against the token-by-token fp64 recurrence.

Tolerances.  bf16 fields: one rounding of an fp32 result, at most 2^-8 of the element: 2^-8
of the norm and of the largest element (the fp32 part is below the rounding of a tie).
fp32: a state remembers 1 / (1 - a) tokens, up to about 3000 for the gates drawn here,
each step rounding by 2^-24 of the state: at most 2e-4 if all errors align, about
sqrt(3000) 2^-24 = 3e-6 if they do not; 2e-5 of the norm and 1e-4 of the largest."""
import numpy as np
import pytest

import _scan_ref as ref
from _util import rel_errors, to_np

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")

BOUND = {"bf16": (2.0 ** -8, 2.0 ** -8), "f32": (2e-5, 1e-4)}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def near(got, want, dtype, what):
    # A factor below fp32's normal range (1 - a at g = 90 is 8e-40) is zero; products with it stay below 2^-120.
    want = np.where(np.abs(want) < 2.0 ** -120, 0.0, want)
    l2, mx = rel_errors(got, want)
    bl, bm = BOUND[dtype]
    assert l2 <= bl and mx <= bm, f"{what}: l2 {l2:.3e} > {bl} or max {mx:.3e} > {bm}"


def fields(B, L, D, dtype, seed, n=3):
    rng = np.random.default_rng(seed)
    out = []
    for k in range(n):
        v = rng.standard_normal((B, L, D))
        if k == 1:
            v = 2.5 + 1.5 * v
        out.append(torch.from_numpy(v).to("cuda", DT[dtype]))
    return out, rng


def run(x, g, dy, leak, h0, dh, lengths):
    B, L, D = x.shape
    y, dx, dg = (torch.full((B, L, D), 7.0, dtype=x.dtype, device="cuda") for _ in range(3))
    state, dh0 = (torch.full((B, D), 7.0, device="cuda") for _ in range(2))
    saved = rlm.scan_saved(B, L, D)
    rlm.rlm_scan_prefill(x, g, y, leak=leak, state_in=h0, state_out=state, saved=saved, lengths=lengths)
    rlm.rlm_scan_backward(dy, x, g, saved, dx, dg, leak=leak, d_state_out=dh, d_state_in=dh0, lengths=lengths)
    torch.cuda.synchronize()
    assert rlm.rlm_get_device_status() == rlm.RLM_OK
    return y, state, dx, dg, dh0


def check(x, g, dy, leak, h0, dh, lengths, dtype):
    got = run(x, g, dy, leak, h0, dh, lengths)
    opt = lambda t: None if t is None else t.cpu().numpy()
    xs, gs, ds = to_np(x), to_np(g), to_np(dy)
    y, state, before = ref.forward(xs, gs, leak, opt(h0), opt(lengths))
    dx, dg, dh0 = ref.backward(ds, xs, gs, leak, before, opt(dh), opt(lengths))
    near(to_np(got[0]), y, dtype, "y")
    near(to_np(got[1]), state, "f32", "state")
    near(to_np(got[2]), dx, dtype, "dx")
    near(to_np(got[3]), dg, dtype, "dg")
    near(to_np(got[4]), dh0, "f32", "d_state_in")
    return got


# One token, lengths about the thread runs (8, 16), the chunk (64) and the tile (128 and up), widths for
# every row layout (8, 16, 32, 64 channels), partial groups, one and several segments.
SHAPES = [(1, 1, 8), (2, 3, 8), (1, 7, 16), (3, 8, 24), (2, 9, 32), (1, 16, 40), (2, 63, 64), (2, 64, 72),
          (1, 65, 128), (3, 127, 64), (1, 128, 200), (1, 129, 8), (5, 500, 8), (2, 1025, 16), (1, 2049, 64),
          (1, 3001, 136), (70, 33, 328), (4, 777, 512), (1, 513, 2048)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("leak", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_gradients(shape, leak, dtype):
    (x, g, dy), rng = fields(*shape, dtype, hash(shape) % 1000)
    B, L, D = shape
    h0 = torch.from_numpy(rng.standard_normal((B, D))).float().cuda()
    dh = torch.from_numpy(rng.standard_normal((B, D))).float().cuda()
    check(x, g, dy, leak, h0, dh, None, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(6, 300, 64), (5, 2050, 8), (3, 1500, 136), (400, 40, 64)])
def test_padding_is_never_read(shape, dtype):
    """Rows of every length, none and all among them; NaN and infinities in the padding."""
    (x, g, dy), rng = fields(*shape, dtype, 5)
    B, L, D = shape
    n = rng.integers(0, L + 1, B)
    n[0], n[1], n[2] = 0, L, 1
    if B > 3:
        n[3], n[4] = -5, L + 9          # clamped
    for k, v in enumerate((float("nan"), float("inf"), float("-inf"))):
        for t in (x, g, dy):
            for b in range(B):
                t[b, max(0, min(L, n[b])) + k::3] = v
    h0 = torch.from_numpy(rng.standard_normal((B, D))).float().cuda()
    dh = torch.from_numpy(rng.standard_normal((B, D))).float().cuda()
    got = check(x, g, dy, True, h0, dh, torch.from_numpy(n).int().cuda(), dtype)
    assert torch.equal(got[1][0], h0[0]) and torch.equal(got[4][0], dh[0])
    assert not got[0][0].any() and not got[2][0].any() and not got[3][0].any()


def test_without_states():
    (x, g, dy), _ = fields(2, 200, 64, "f32", 9)
    check(x, g, dy, False, None, None, None, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,L,D", [(2, 700, 64), (1, 1, 8), (3, 130, 24)])
def test_views_of_a_projection(B, L, D, dtype):
    """x and g as halves of one buffer, dx and dg likewise, y into a slice of a wider one, time-major dy."""
    (f, _, dy), rng = fields(B, L, 2 * D, dtype, 3)
    f[..., D:] += 2
    dy = dy[..., :D].transpose(0, 1).contiguous().transpose(0, 1)          # [L][B][D] in memory
    x, g = f[..., :D], f[..., D:]
    base = run(x.contiguous(), g.contiguous(), dy.contiguous(), True, None, None, None)
    d = torch.full((B, L, 2 * D), 7.0, dtype=x.dtype, device="cuda")
    wide = torch.full((B, L, 3 * D), 7.0, dtype=x.dtype, device="cuda")
    saved = rlm.scan_saved(B, L, D)
    rlm.rlm_scan_prefill(x, g, wide[..., D:2 * D], saved=saved)
    rlm.rlm_scan_backward(dy, x, g, saved, d[..., :D], d[..., D:])
    assert torch.equal(wide[..., D:2 * D], base[0])
    assert torch.equal(d[..., :D], base[2]) and torch.equal(d[..., D:], base[3])
    assert (wide[..., :D] == 7).all() and (wide[..., 2 * D:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("leak", [True, False])
@pytest.mark.parametrize("B,D", [(1, 8), (3, 72), (64, 1024), (7, 4104)])
def test_decode(B, D, leak, dtype):
    (x, g, _), rng = fields(B, 5, D, dtype, 21)
    state = torch.from_numpy(rng.standard_normal((B, D))).float().cuda()
    want, end, _ = ref.forward(to_np(x), to_np(g), leak, state.cpu().numpy())
    y = torch.empty(B, 5, D, dtype=x.dtype, device="cuda")
    for t in range(5):
        rlm.rlm_scan_decode(x[:, t], g[:, t], state, y[:, t], leak=leak)
    near(to_np(y), want, dtype, "y")
    near(to_np(state), end, "f32", "state")


def test_continued_prefill_and_decode_agree_with_one_prefill():
    (x, g, _), _ = fields(2, 301, 64, "f32", 4)
    y, s = torch.empty_like(x), torch.empty(2, 64, device="cuda")
    rlm.rlm_scan_prefill(x, g, y, state_out=s)
    z, st = torch.empty_like(x), torch.zeros(2, 64, device="cuda")
    rlm.rlm_scan_prefill(x[:, :100], g[:, :100], z[:, :100], state_in=st, state_out=st)
    rlm.rlm_scan_prefill(x[:, 100:300], g[:, 100:300], z[:, 100:300], state_in=st, state_out=st)
    rlm.rlm_scan_decode(x[:, 300], g[:, 300], st, z[:, 300])
    near(to_np(z), to_np(y), "f32", "y")
    near(to_np(st), to_np(s), "f32", "state")


def test_extreme_gates():
    """sigma saturates at both ends without NaN: +inf keeps the state, -inf forgets it."""
    (x, _, dy), rng = fields(1, 200, 64, "f32", 2)
    g = torch.from_numpy(rng.choice([-200.0, -90.0, 90.0, 200.0, np.inf, -np.inf], (1, 200, 64))).float().cuda()
    check(x, g, dy, True, None, None, None, "f32")


@pytest.mark.parametrize("B,L,D", [(1, 4096, 64), (4, 4096, 256), (1, 40000, 8)])
def test_repeats_bit_for_bit_and_on_another_stream(B, L, D):
    """Segmented launches: the exchange's order is fixed."""
    (x, g, dy), rng = fields(B, L, D, "bf16", 8)
    dh = torch.from_numpy(rng.standard_normal((B, D))).float().cuda()
    first = run(x, g, dy, True, None, dh, None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            again = run(x, g, dy, True, None, dh, None)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_graph_replays():
    """A captured call may be replayed with new inputs."""
    (x, g, dy), _ = fields(1, 4096, 64, "f32", 8)
    y = torch.empty_like(x)
    rlm.rlm_scan_prefill(x, g, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rlm.rlm_scan_prefill(x, g, y)
    for k in range(3):
        x.copy_(torch.randn_like(x))
        graph.replay()
        want = torch.empty_like(x)
        rlm.rlm_scan_prefill(x, g, want)
        assert torch.equal(y, want)


def test_gradients_against_differences():
    """Central differences of the fp64 definition: the formulas themselves, then the kernels against them."""
    (x, g, dy), rng = fields(1, 12, 8, "f32", 31)
    h0, dh = rng.standard_normal((1, 8)), rng.standard_normal((1, 8))
    xs, gs, ds = to_np(x), to_np(g), to_np(dy)
    for leak in (True, False):
        def loss(xv, gv, hv):
            y, s, _ = ref.forward(xv, gv, leak, hv)
            return (y * ds).sum() + (s * dh).sum()
        eps = 1e-6

        def grad(which):
            args = [xs, gs, h0]
            out = np.zeros_like(args[which])
            for i in np.ndindex(out.shape):
                v = [a.copy() for a in args]
                v[which][i] += eps
                up = loss(*v)
                v[which][i] -= 2 * eps
                out[i] = (up - loss(*v)) / (2 * eps)
            return out
        f = lambda a: torch.from_numpy(a).float().cuda()
        got = run(x, g, dy, leak, f(h0), f(dh), None)
        for k, w in ((2, 0), (3, 1), (4, 2)):
            l2, mx = rel_errors(to_np(got[k]), grad(w))
            assert l2 < 1e-5 and mx < 1e-5, (leak, k, l2, mx)


def test_long_strides():
    """Offsets past 2^31 elements: the rows of a sequence spread over a wide buffer."""
    B, L, D, pitch = 1, 9, 64, 1 << 28
    try:
        big = torch.zeros(L * pitch, dtype=torch.bfloat16, device="cuda")
    except torch.cuda.OutOfMemoryError:
        pytest.skip("no room for a 4.8 GB buffer")
    (x, g, _), _ = fields(B, L, D, "bf16", 6)
    at = big.as_strided((B, L, D), (L * pitch, pitch, 1))
    at.copy_(x)
    y, z = torch.empty_like(x), torch.empty_like(x)
    rlm.rlm_scan_prefill(x, g, y)
    rlm.rlm_scan_prefill(at, g, z)
    assert torch.equal(y, z)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_inputs_shared_by_the_batch(dtype):
    """A batch stride of zero: every row reads the same drive (or gate)."""
    (x, g, dy), _ = fields(3, 150, 64, dtype, 12)
    one = x[:1].expand(3, -1, -1)
    want = run(one.contiguous(), g, dy, True, None, None, None)
    got = run(one, g, dy, True, None, None, None)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = run(x, g[:1].expand(3, -1, -1), dy, True, None, None, None)
    want = run(x, g[:1].expand(3, -1, -1).contiguous(), dy, True, None, None, None)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
