"""The AdamW step against its fp64 definition.

Tolerances.  fp32 moments: two products and a sum, at most 3 * 2^-24 of the terms; the weight:
a dozen roundings of a step that is small against it, and one of the weight; 1e-6 of the norm
and of the largest (2^-20) covers both.  bf16 weights: one rounding, 2^-8.  8-bit codes have 4
significant bits, so a value is within 2^-4 of itself, or within half the smallest code
2^-10 of its block's scale; sqrt(v) at the smallest code is up to a whole one off."""
import numpy as np
import pytest

from _util import rel_errors

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HP = dict(beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


def near(got, want, bound, what):
    l2, mx = rel_errors(got.double().cpu().numpy(), np.asarray(want))
    assert l2 <= bound and mx <= bound, f"{what}: l2 {l2:.3e}, max {mx:.3e} > {bound:.1e}"


def step64(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay):
    m = m + (1 - beta1) * (g - m)
    v = v + (1 - beta2) * (g * g - v)
    p = p - lr * weight_decay * p - lr * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return p, m, v


def tensors(sizes, param, grad, bits, master, seed, offset=0):
    """Weights and gradients of the given sizes; ``offset``: values that every buffer starts past alignment."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda n: torch.randn(n + offset, generator=gen, device="cuda")
    out = []
    for n in sizes:
        full = 0.05 * rn(n)
        grow = torch.exp(3 * torch.randn(n + offset, generator=gen, device="cuda")) * 1e-3
        p, g = full.to(DT[param])[offset:], (rn(n) * grow).to(DT[grad])[offset:]
        st = rlm.AdamState.zeros(p, bits)
        if offset:
            dt = st.m.dtype
            st.m, st.v = (torch.zeros(n + offset, dtype=torch.uint8 if bits == 8 else dt, device="cuda")[offset:].view(dt)
                          for _ in range(2))
        out.append((p, g, st, full[offset:] if master else None))
    return out


SIZES = [[1], [7], [256], [2048, 2049, 255], [5, 100003, 1, 4096, 31], list(range(1, 900, 2))]
KINDS = [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "bf16", False), ("bf16", "bf16", True),
         ("bf16", "f32", True)]


@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sizes", SIZES, ids=len)
def test_three_steps_with_32_bit_moments(sizes, kind, offset):
    param, grad, master = kind
    ts = tensors(sizes, param, grad, 32, master, 1, offset)
    group = rlm.AdamGroup([t[0] for t in ts], [t[1] for t in ts], [t[2] for t in ts], [t[3] for t in ts] if master else None)
    cat = lambda k: torch.cat([k(t).reshape(-1) for t in ts])
    for t in (1, 2, 3):
        for _, g, _, _ in ts:
            g.mul_(-0.7)
        old = [cat(lambda t: t[3] if master else t[0]), cat(lambda t: t[1]), cat(lambda t: t[2].m), cat(lambda t: t[2].v)]
        want, m, v = step64(*(o.double().cpu().numpy() for o in old), t, 1e-2, **HP)
        rlm.rlm_adamw_step(group, t, 1e-2, **HP)
        near(cat(lambda t: t[2].m), m, 1e-6, "m")
        near(cat(lambda t: t[2].v), v, 1e-6, "v")
        near(cat(lambda t: t[0]), want, 1e-6 if param == "f32" else 2.0 ** -8, "weight")
        if master:
            near(cat(lambda t: t[3]), want, 1e-6, "master")
            assert all(torch.equal(p, w.bfloat16()) for p, _, _, w in ts)


def blocks(x):
    n = -(-x.size // 256) * 256
    return np.pad(x, (0, n - x.size)).reshape(-1, 256)


@pytest.mark.parametrize("offset", [0, 5])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sizes", SIZES, ids=len)
def test_8_bit_moments(sizes, kind, offset):
    """Each step from the moments as they are kept; what is kept afterwards is the new moments, rounded."""
    param, grad, master = kind
    ts = tensors(sizes, param, grad, 8, master, 2, offset)
    group = rlm.AdamGroup([t[0] for t in ts], [t[1] for t in ts], [t[2] for t in ts], [t[3] for t in ts] if master else None)
    for step in (1, 2, 3):
        ref = []
        for p, g, st, w in ts:
            g.mul_(-1.3)
            m, v = (t.double().cpu().numpy() for t in st.values())
            ref.append(step64((w if master else p).double().cpu().numpy(), g.double().cpu().numpy(), m, v, step, 1e-2, **HP))
        rlm.rlm_adamw_step(group, step, 1e-2, **HP)
        for (p, g, st, w), (rp, rm, rv) in zip(ts, ref):
            near(w if master else p, rp, 1e-6 if master or param == "f32" else 2.0 ** -8, "weight")
            for code, scale, val, smallest in ((st.m, st.m_scale, rm, 0.5), (st.v, st.v_scale, np.sqrt(rv), 1.0)):
                top = np.abs(blocks(val)).max(1)
                s = scale.double().cpu().numpy()
                # The largest value of a block is in [128, 256) times its scale (a value at a power of two may fall
                # either side).
                assert ((top < 256.001 * s) & (top > 127.999 * s)).all()
                got = blocks(code.double().cpu().numpy()) * s[:, None]
                off = np.abs(got - blocks(val))
                assert (off <= np.maximum(np.abs(blocks(val)) * 2.0 ** -4 * 1.0001, smallest * 2.0 ** -9 * s[:, None] * 1.0001)).all()
            assert ((st.v.float() > 0).cpu().numpy() == (rv > 0)).all()


def test_a_zero_gradient_and_zero_blocks():
    for bits in (8, 32):
        (p, g, st, _), = tensors([700], "f32", "f32", bits, False, 3)
        g.zero_()
        old = p.clone()
        rlm.rlm_adamw_step(rlm.AdamGroup([p], [g], [st]), 1, 1e-2, **HP)
        assert torch.equal(p, old * np.float32(1 - 1e-3))
        m, v = st.values()
        assert not m.any() and not v.any() and torch.isfinite(p).all()


def test_tiny_and_huge_gradients_stay_finite():
    for bits in (8, 32):
        (p, g, st, _), = tensors([512], "f32", "f32", bits, False, 3)
        g[:256] = 1e-30
        g[256:] = 1e15
        rlm.rlm_adamw_step(rlm.AdamGroup([p], [g], [st]), 1, 1e-2, **HP)
        assert torch.isfinite(p).all() and all(torch.isfinite(t).all() for t in st.values())


def test_gradient_scale():
    a, b, c = (tensors([1000], "f32", "f32", 32, False, 4)[0] for _ in range(3))
    b[1].mul_(4)
    rlm.rlm_adamw_step(rlm.AdamGroup([a[0]], [a[1]], [a[2]]), 1, 1e-2, **HP)
    rlm.rlm_adamw_step(rlm.AdamGroup([b[0]], [b[1]], [b[2]]), 1, 1e-2, grad_scale=torch.tensor(0.25, device="cuda"), **HP)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2].v, b[2].v)
    old = c[0].clone()
    for bad in (float("inf"), float("nan")):
        rlm.rlm_adamw_step(rlm.AdamGroup([c[0]], [c[1]], [c[2]]), 1, 1e-2, grad_scale=torch.tensor(bad, device="cuda"), **HP)
    assert torch.equal(c[0], old) and not c[2].m.any()


def test_more_tensors_than_a_launch_holds():
    before = rlm.rlm_kernels_launched()
    ts = tensors([3] * 1001, "f32", "f32", 32, False, 5)
    one = tensors([3] * 1001, "f32", "f32", 32, False, 5)
    rlm.rlm_adamw_step(rlm.AdamGroup([t[0] for t in ts], [t[1] for t in ts], [t[2] for t in ts]), 1, 1e-2, **HP)
    assert rlm.rlm_kernels_launched() - before == 3
    for k in (0, 399, 400, 799, 800, 1000):
        rlm.rlm_adamw_step(rlm.AdamGroup([one[k][0]], [one[k][1]], [one[k][2]]), 1, 1e-2, **HP)
        assert torch.equal(one[k][0], ts[k][0])


def test_a_tensor_past_2_31_values():
    n = (1 << 31) + 77
    if torch.cuda.mem_get_info()[0] < 9 * n:
        pytest.skip("no room for a tensor of 2^31 values")
    p = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    st = rlm.AdamState.zeros(p, 8)
    rlm.rlm_adamw_step(rlm.AdamGroup([p], [g], [st]), 1, 0.25, **HP)
    assert (p[-100:] == p[0]).all() and p[0] != 1 and (st.m[-100:].float() == st.m[:1].float()).all()


def test_python_checks():
    (p, g, st, _), = tensors([100], "f32", "f32", 32, False, 6)
    for args in (([], [], []), ([p], [g[:50]], [st]), ([p], [g.double()], [st]), ([p[::2]], [g[:50]], [st]),
                 ([p], [g], [rlm.AdamState.zeros(p[:50])]), ([p], [g], [st], [p, p])):
        with pytest.raises(ValueError):
            rlm.AdamGroup(*args)
    with pytest.raises(ValueError):
        rlm.AdamState.zeros(p, 4)
    with pytest.raises(rlm.RlmError):
        rlm.rlm_adamw_step(rlm.AdamGroup([p], [g], [st]), 0, 1e-3)
