"""The operators together: a stack of gated recurrent blocks learns, its gradients are those of
the fp64 definition, and decoding continues a padded prefill."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import gated_block  # noqa: E402


@pytest.mark.parametrize("bits", [32, 8])
def test_the_example_learns_and_decodes(bits):
    first, last, worst = gated_block.main(steps=120, bits=bits, B=4, L=128, quiet=True)
    assert last < 0.5 * first
    # Outputs are a few units; prefill and decode round x, g and s to bf16 at the same places.
    assert worst < 0.1


def test_block_gradients_against_fp64():
    """One block's weight and input gradients against autograd through the definition in fp64.  The
    intermediate fields are rounded to bf16 (2^-8 each) on the way forward and back: 3 % of the norm."""
    D, B, L = 64, 2, 70
    block = gated_block.Block(D, torch.Generator(device="cuda").manual_seed(3))
    gen = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn(B, L, D, generator=gen, device="cuda").bfloat16()
    d = torch.randn(B, L, D, generator=gen, device="cuda").bfloat16()
    out = block.forward(h)
    dh = block.backward(d)
    h64, wi, bi, wo = (t.double().requires_grad_() for t in (h, block.w_in, block.b_in, block.w_out))
    p = h64 @ wi.T + bi
    a, x = torch.sigmoid(p[..., D:]), p[..., :D]
    s, st = [], torch.zeros(B, D, dtype=torch.float64, device="cuda")
    for t in range(L):
        st = a[:, t] * st + (1 - a[:, t]) * x[:, t]
        s.append(st)
    y = torch.stack(s, 1) @ wo.T + h64
    y.backward(d.double())
    for got, want, name in ((out, y, "out"), (dh, h64.grad, "dh"), (block.grads["w_in"], wi.grad, "w_in"),
                            (block.grads["b_in"], bi.grad, "b_in"), (block.grads["w_out"], wo.grad, "w_out")):
        rel = ((got.double() - want).norm() / want.norm()).item()
        assert rel < 0.03, (name, rel)
