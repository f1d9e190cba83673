"""The linear layer and its gradients against fp64 products of the same bf16 inputs.

Tolerances.  Inputs are bf16 and exact; sums are fp32, so the result differs by its one
rounding to bf16 (8 significant bits), at most 2^-8 of the element: 2^-8 of the norm and of
the largest element.  dx and dw of a layer with an activation see dz rounded to bf16 as
well: with one term in the sum the two roundings add, 2^-7.  The fp32 outputs (dw kept in
fp32, dbias) have only the sums' errors: the tensor cores add products of a 16-long step and
then to the accumulator, each addition within 2^-23 of the sum of the terms' magnitudes;
sums of n random terms have magnitude sqrt(n) against n, so sqrt(n) 2^-23 n / 16 steps'
worth at most: 2e-4 of the norm at n = 2000, met with room."""
import numpy as np
import pytest

from _util import rel_errors

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")

B16 = 2.0 ** -8
ACTS = ["none", "silu", "gelu", "sigmoid"]


def act64(z, kind):
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "sigmoid":
        return torch.sigmoid(z)
    return torch.nn.functional.gelu(z, approximate="tanh") if kind == "gelu" else z


def near(got, want, bound, what):
    l2, mx = rel_errors(got.double().cpu().numpy(), want.double().cpu().numpy())
    assert l2 <= bound and mx <= bound, f"{what}: l2 {l2:.3e}, max {mx:.3e} > {bound:.1e}"


def make(R, K, N, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return (rn(R, K).bfloat16(), (rn(N, K) * K ** -0.5).bfloat16(), 0.5 * rn(N), rn(R, N).bfloat16(),
            rn(R, N).bfloat16())


def done():
    torch.cuda.synchronize()
    assert rlm.rlm_get_device_status() == rlm.RLM_OK


# One row, rows about the tile's 128 and the few-row forms, contractions about the step of 64, columns about
# 128 and 256, products of few tiles (cut along the contraction) and of many.
SHAPES = [(1, 8, 8), (1, 4096, 1000), (2, 72, 16), (5, 64, 256), (8, 2048, 512), (16, 136, 264), (17, 1024, 40),
          (33, 512, 1032), (64, 200, 128), (127, 64, 8), (128, 128, 256), (129, 520, 136), (200, 4096, 256),
          (257, 8, 512), (300, 1000, 3000), (1000, 264, 2048), (4099, 256, 512), (20000, 128, 384), (515, 8192, 1024)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", ACTS)
def test_forward(shape, act):
    R, K, N = shape
    x, w, bias, res, _ = make(R, K, N)
    z = x.double() @ w.double().T
    for b, r in ((None, None), (bias, res)):
        y, pre = (torch.full((R, N), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        rlm.rlm_linear(x, w, y, bias=b, residual=r, act=act, pre=pre)
        done()
        want = z if b is None else z + b.double()
        near(pre, want, B16, "pre")
        want = act64(want, act)
        near(y, want if r is None else want + r.double(), B16, "y")
        only = torch.full_like(y, 7.0)
        rlm.rlm_linear(x, w, only, bias=b, residual=r, act=act)
        assert torch.equal(only, y)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", ACTS)
def test_gradients(shape, act):
    R, K, N = shape
    x, w, _, pre, dy = make(R, K, N, 1)
    d = dy.double()
    if act != "none":
        z = pre.double().requires_grad_()
        d, = torch.autograd.grad(act64(z, act), z, d)
    dx, dw = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
    db, dwf = torch.full((N,), 7.0, device="cuda"), torch.full((N, K), 7.0, device="cuda")
    p = pre if act != "none" else None
    rlm.rlm_linear_backward(dy, x, w, dx=dx, dw=dw, dbias=db, act=act, pre=p)
    rlm.rlm_linear_backward(dy, x, w, dw=dwf, act=act, pre=p)
    done()
    near(dx, d @ w.double(), B16 if act == "none" else 2 * B16, "dx")
    near(dw, d.T @ x.double(), B16 if act == "none" else 2 * B16, "dw")
    near(dwf, d.T @ x.double(), 2e-4 if act == "none" else B16, "dw in fp32")
    near(db, d.sum(0), 2e-5, "dbias")


def test_each_gradient_alone():
    x, w, _, pre, dy = make(200, 64, 72)
    want = [torch.empty_like(x), torch.empty_like(w), torch.empty(72, device="cuda")]
    rlm.rlm_linear_backward(dy, x, w, *want, act="silu", pre=pre)
    for k, name in enumerate(("dx", "dw", "dbias")):
        got = torch.full_like(want[k], 7.0)
        rlm.rlm_linear_backward(dy, x, w, **{name: got}, act="silu", pre=pre)
        assert torch.equal(got, want[k]), name


@pytest.mark.parametrize("R", [3, 150, 1000])
def test_views_and_a_residual_in_place(R):
    """Row pitches wider than the rows on every matrix; leading dimensions; neighbours untouched."""
    K, N = 72, 136
    x, w, bias, res, dy = make(R, K, N)
    wide = lambda t, at, n: torch.full((t.shape[0], n), 7.0, dtype=t.dtype, device="cuda").index_copy_(
        1, torch.arange(at, at + t.shape[1], device="cuda"), t)
    X, W, Y, G = wide(x, 8, 96), wide(w, 0, 80), wide(res, 16, 176), wide(dy, 24, 200)
    xv, wv, yv, gv = X[:, 8:8 + K], W[:, :K], Y[:, 16:16 + N], G[:, 24:24 + N]
    want = torch.empty(R, N, dtype=torch.bfloat16, device="cuda")
    rlm.rlm_linear(x, w, want, bias=bias, residual=res, act="gelu")
    rlm.rlm_linear(xv, wv, yv, bias=bias, residual=yv, act="gelu")
    assert torch.equal(yv, want)
    assert (Y[:, :16] == 7).all() and (Y[:, 16 + N:] == 7).all()
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    rlm.rlm_linear_backward(dy, x, w, dx=dx, dw=dw)
    both = torch.full((R, 2 * K + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    rlm.rlm_linear_backward(gv, xv, wv, dx=both[:, 8:8 + K])
    assert torch.equal(both[:, 8:8 + K], dx) and (both[:, 8 + K:] == 7).all() and (both[:, :8] == 7).all()
    dwv = torch.full((N, K + 8), 7.0, device="cuda")
    rlm.rlm_linear_backward(gv, xv, wv, dw=dwv[:, :K])
    assert torch.equal(dwv[:, :K].bfloat16(), dw) and (dwv[:, K:] == 7).all()
    y3 = torch.empty(R, 1, N, dtype=torch.bfloat16, device="cuda")
    rlm.rlm_linear(x[:, None], w, y3, bias=bias, residual=res[:, None], act="gelu")
    assert torch.equal(y3[:, 0], want)


def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph():
    x, w, bias, res, dy = make(300, 2048, 512)
    y = torch.empty(300, 512, dtype=torch.bfloat16, device="cuda")
    dw = torch.empty_like(w)
    rlm.rlm_linear(x, w, y, bias=bias, residual=res)
    rlm.rlm_linear_backward(dy, x, w, dw=dw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y2, dw2 = torch.empty_like(y), torch.empty_like(w)
        rlm.rlm_linear(x, w, y2, bias=bias, residual=res)
        rlm.rlm_linear_backward(dy, x, w, dw=dw2)
    side.synchronize()
    assert torch.equal(y, y2) and torch.equal(dw, dw2)
    ws = torch.empty(max(1, rlm.rlm_linear_workspace_size(300, 2048, 512)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rlm.rlm_linear(x, w, y2, bias=bias, residual=res, workspace=ws)
    x.mul_(-1)
    graph.replay()
    rlm.rlm_linear(x, w, y, bias=bias, residual=res)
    torch.cuda.synchronize()
    assert torch.equal(y, y2)


def test_infinities_and_nan_stay_in_their_rows():
    x, w, _, _, _ = make(130, 64, 64)
    x[3, 5], x[129, 63] = float("inf"), float("nan")
    y = torch.empty(130, 64, dtype=torch.bfloat16, device="cuda")
    rlm.rlm_linear(x, w, y)
    bad = ~torch.isfinite(y).all(1)
    assert bad[3] and bad[129] and bad.sum() == 2
    big = torch.tensor([[300.0, -300.0, 3e4, -3e4, 0.0, -0.0, 1e-3, -1e-3]], device="cuda").bfloat16()
    eye = torch.eye(8, device="cuda").bfloat16()
    for act in ACTS:
        y = torch.empty(1, 8, dtype=torch.bfloat16, device="cuda")
        rlm.rlm_linear(big, eye, y, act=act)
        near(y, act64(big.double(), act), B16, act)
        dx = torch.empty_like(big)
        rlm.rlm_linear_backward(torch.ones_like(big), big, eye, dx=dx, act=act, pre=big if act != "none" else None)
        z = big.double().requires_grad_()
        want, = torch.autograd.grad(act64(z, act).sum(), z)
        near(dx, want, 2 * B16, act)


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_gradients_against_differences(act):
    """dx and dw against central differences of the fp64 definition (inputs exact in bf16)."""
    x, w, _, _, dy = make(3, 8, 8, 3)
    xs, ws, ds = x.double(), w.double(), dy.double()
    pre = torch.empty(3, 8, dtype=torch.bfloat16, device="cuda")
    rlm.rlm_linear(x, w, torch.empty_like(pre), act=act, pre=pre)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    rlm.rlm_linear_backward(dy, x, w, dx=dx, dw=dw, act=act, pre=pre)
    loss = lambda a, b: (act64(a @ b.T, act) * ds).sum().item()
    for got, which in ((dx, 0), (dw, 1)):
        want = torch.zeros_like((xs, ws)[which])
        for i in np.ndindex(*want.shape):
            v = [xs.clone(), ws.clone()]
            v[which][i] += 1e-6
            up = loss(*v)
            v[which][i] -= 2e-6
            want[i] = (up - loss(*v)) / 2e-6
        # pre's own rounding moves act' by at most 2^-8 |z| |act''| (below 2^-8 here) beside dz's and the result's.
        near(got, want, 3 * B16, act)


def test_offsets_past_2_31_elements():
    """Rows of y (and of dy, dx) beyond 2^31 elements, against the same rows by themselves."""
    R, K, N = 530000, 8, 4104
    if torch.cuda.mem_get_info()[0] < 3 * 2 * R * N:
        pytest.skip("no room for fields of 2^31 elements")
    x = torch.randn(R, K, device="cuda").bfloat16()
    w = torch.randn(N, K, device="cuda").bfloat16()
    y = torch.empty(R, N, dtype=torch.bfloat16, device="cuda")
    rlm.rlm_linear(x, w, y, act="silu")
    tail = torch.empty(300, N, dtype=torch.bfloat16, device="cuda")
    rlm.rlm_linear(x[-300:], w, tail, act="silu")
    assert torch.equal(y[-300:], tail)
    dx, part = torch.empty_like(x), torch.empty(300, K, dtype=torch.bfloat16, device="cuda")
    rlm.rlm_linear_backward(y, x, w, dx=dx)
    rlm.rlm_linear_backward(y[-300:], x[-300:], w, dx=part)
    near(dx[-300:], y[-300:].double() @ w.double(), B16, "dx")
    near(part, y[-300:].double() @ w.double(), B16, "dx of the tail")


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_slopes_of_extreme_pre_activations(act):
    """act'(z) over all of bf16's range: its limits far out, NaN of NaN.  One row, so that dbias is dz
    itself.  Bound: the approximate instructions on arguments up to 128 (2^-15), and 1e-30 where the
    slope itself is nothing."""
    mags = [0.0, 1e-30, 1e-3, 0.5, 1.0, 3.0, 5.0, 8.0, 9.5, 10.5, 20.0, 60.0, 84.0, 90.0, 300.0, 1e4, 1e9, 1e13, 1e20,
            3e38, float("inf")]
    z = torch.tensor([s * m for m in mags for s in (1, -1)] + [float("nan")] * 6).bfloat16().cuda()
    N = z.numel()
    x, w = torch.zeros(1, 8, device="cuda").bfloat16(), torch.zeros(N, 8, device="cuda").bfloat16()
    got = torch.empty(N, device="cuda")
    rlm.rlm_linear_backward(torch.ones(1, N, device="cuda").bfloat16(), x, w, pre=z[None], act=act, dbias=got)
    done()
    z64 = z.double().clamp(-400, 400)
    bend = 2 * (2 / np.pi) ** 0.5
    u = bend * (z64 + 0.044715 * z64 ** 3) if act == "gelu" else z64
    slope = bend * z64 * (1 + 3 * 0.044715 * z64 ** 2) if act == "gelu" else z64
    s, rest = torch.sigmoid(u), torch.sigmoid(-u)           # (1 - s would lose rest)
    want = s * rest if act == "sigmoid" else s * (1 + slope * rest)
    assert torch.isnan(got[-6:]).all()
    assert ((got.double() - want)[:-6].abs() <= 2.0 ** -15 * want[:-6].abs() + 1e-30).all()


def test_workspace_belongs_to_the_stream_of_the_call():
    """A call's own workspace is not handed to the current stream while the call's stream uses it."""
    R, K, N = 515, 8192, 1024
    x, w, _, _, dy = make(R, K, N)
    size = rlm.rlm_linear_workspace_size(R, K, N)
    assert size > 0
    want, got = torch.empty_like(dy), torch.empty_like(dy)
    rlm.rlm_linear(x, w, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        torch.cuda.empty_cache()
        with torch.cuda.stream(side):
            torch.cuda._sleep(4_000_000)
        rlm.rlm_linear(x, w, got, stream=stream)
        other = torch.empty(size, dtype=torch.uint8, device="cuda")
        for _ in range(1500):                   # on the current stream, while the call runs
            other.fill_(255)
        done()
        assert torch.equal(got, want)


@pytest.mark.parametrize("shape", [(8000, 2048, 1160), (16387, 1160, 2056), (4096, 4096, 4096)])
def test_last_round_of_tiles_in_halves(shape):
    """Products whose last round of 256 x 256 tiles is cut into halves, some with few columns."""
    R, K, N = shape
    x, w, bias, res, dy = make(R, K, N)
    y, pre = torch.empty_like(dy), torch.empty_like(dy)
    rlm.rlm_linear(x, w, y, bias=bias, residual=res, act="silu", pre=pre)
    z = x.double() @ w.double().T + bias.double()
    near(pre, z, B16, "pre")
    near(y, act64(z, "silu") + res.double(), B16, "y")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    rlm.rlm_linear_backward(dy, x, w, dx=dx, dw=dw)
    done()
    near(dx, dy.double() @ w.double(), B16, "dx")
    near(dw, dy.double().T @ x.double(), B16, "dw")
