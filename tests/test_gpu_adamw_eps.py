"""AdamW's eps down to the smallest numbers: where both moments are zero, so is the step."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [1e-45, 1e-42, 1e-39, 1.1e-38, 1.2e-38, 1e-30, 1e-8])
def test_zero_moments_leave_the_weight(eps, bits):
    gen = torch.Generator(device="cuda").manual_seed(0)
    p, g = torch.randn(600, generator=gen, device="cuda"), torch.randn(600, generator=gen, device="cuda")
    g[::3] = 0
    old = p.clone()
    rlm.rlm_adamw_step(rlm.AdamGroup([p], [g], [rlm.AdamState.zeros(p, bits)]), 1, 0.125, eps=eps, weight_decay=0.0)
    assert torch.equal(p[::3], old[::3])
    # The first step is lr times the gradient's sign; a few of fp32's last bits on the way.
    want = old.double() - 0.125 * torch.sign(g).double() * (g.abs() / (g.abs() + eps)).nan_to_num().double()
    assert ((p.double() - want).abs() <= 2.0 ** -20 * (old.abs() + 0.125)).all()
