"""Kernels that may be resident before the ones ahead of them end read what those write.

Every step below follows a kernel that still writes the step's inputs when the step is enqueued: the
result is compared bit for bit with the same two calls with a synchronisation in between."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")

BF16 = torch.bfloat16


def both(restore, write, read, outputs, repeats=20):
    """write then read, at once and with a synchronisation between, from the same start."""
    for _ in range(repeats):
        got = []
        for wait in (True, False):
            restore()
            torch.cuda.synchronize()
            write()
            if wait:
                torch.cuda.synchronize()
            read()
            torch.cuda.synchronize()
            got.append([t.clone() for t in outputs])
        assert all(torch.equal(a, b) for a, b in zip(*got))
    assert all(torch.isfinite(t).all() for t in got[0])


# One block per batch row (coupled), the recurrence step and a finishing kernel (coupled, wide rows; modes
# that are no power of two), the plain mixer step.
@pytest.mark.parametrize("D,M,K,H", [(256, 16, 4, 8), (512, 8, 3, 16), (1024, 16, 4, 8), (64, 12, 4, 4), (256, 16, 4, 0),
                                     (64, 7, 4, 0)])
def test_a_mixer_step_right_after_its_weights_are_updated(D, M, K, H):
    """An AdamW step of about 0.2 ms whose last tensors are the mixer's weights, then a decode step."""
    B = 8
    gen = torch.Generator(device="cuda").manual_seed(D + M)
    rn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    c_raw = rn(max(H, 1), max(H, 1))
    local = rlm.Local(rn(D, K), rn(D))
    big = rn(40_000_000)
    ws = [big, local.conv_w, local.scale, c_raw]
    states = [rlm.AdamState.zeros(w) for w in ws]
    group = rlm.AdamGroup(ws, [rn(*w.shape) for w in ws], states)
    old = [w.clone() for w in ws[1:]]
    st = rlm.State.empty(B, D, M)
    rlm.rlm_state_init(st, rlm.Params(*(0.5 + 0.1 * rn(D, M).abs() for _ in range(4))))
    s0, u0 = rn(B, D, M, 2), rn(B, K - 1, D).to(BF16)
    conv = rlm.ConvState(u0.clone())
    x, g, z = rn(B, D).to(BF16), rn(B, D).to(BF16), torch.empty(B, D, dtype=BF16, device="cuda")

    def restore():
        for w, o, m in zip(ws[1:], old, states[1:]):
            w.copy_(o)
            m.m.zero_()
            m.v.zero_()
        st.s.copy_(s0)
        conv.u.copy_(u0)
        z.fill_(7)

    both(restore, lambda: rlm.rlm_adamw_step(group, 1, 0.5),
         lambda: rlm.rlm_mixer_decode(x, g, st, local, conv, z, coupling=rlm.Coupling(c_raw, 0.7) if H else None),
         (z, st.s, conv.u))


@pytest.mark.parametrize("M", [16, 7])
def test_a_decode_step_right_after_its_token_is_written(M):
    """The token comes from a product of many tiles that ends while the step is resident."""
    B, K, D = 64, 8192, 4096
    gen = torch.Generator(device="cuda").manual_seed(M)
    rn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    h, w = rn(2048, K).to(BF16), (rn(D, K) * K ** -0.5).to(BF16)
    x = torch.zeros(2048, D, dtype=BF16, device="cuda")
    st = rlm.State.empty(B, D, M)
    rlm.rlm_state_init(st, rlm.Params(*(0.5 + 0.1 * rn(D, M).abs() for _ in range(4))))
    s0, y = rn(B, D, M, 2), torch.empty(B, D, dtype=BF16, device="cuda")

    def restore():
        x.zero_()
        st.s.copy_(s0)

    both(restore, lambda: rlm.rlm_linear(h, w, x), lambda: rlm.rlm_mix_decode(x[-B:], st, y), (y, st.s))
