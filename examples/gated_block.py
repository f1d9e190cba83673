"""Trains a small stack of gated recurrent blocks and decodes with it, on one GPU.

    block   p = h w_in^T + b_in;  (x | g) = halves of p;  s = gated recurrence of (x, g)
            h' = s w_out^T + h

The task: from noise u_t, predict a running average of it (a state that only a recurrence
with a learned decay can hold).  Every product, scan and optimizer step is one of the
library's calls; PyTorch holds the memory and forms the loss.

    python examples/gated_block.py [--steps 200] [--bits 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_05583_gb300 as rlm  # noqa: E402

BF16 = torch.bfloat16


class Block:
    """One block: its weights, their gradients and the buffers of a training pass."""

    def __init__(self, D: int, gen: torch.Generator):
        randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
        self.D = D
        self.w_in = (randn(2 * D, D) * D ** -0.5).to(BF16)
        self.b_in = torch.cat([torch.zeros(D, device="cuda"), 2 + randn(D)])       # gates start near 0.9
        self.w_out = (randn(D, D) * 0.3 * D ** -0.5).to(BF16)
        self.grads = {k: torch.zeros_like(getattr(self, k)) for k in ("w_in", "b_in", "w_out")}

    def forward(self, h: torch.Tensor, lengths: torch.Tensor | None = None) -> torch.Tensor:
        B, L, D = h.shape
        p = torch.empty(B, L, 2 * D, dtype=BF16, device="cuda")
        rlm.rlm_linear(h, self.w_in, p, bias=self.b_in)
        s, saved = torch.empty_like(h), rlm.scan_saved(B, L, D)
        self.state = torch.empty(B, D, device="cuda")
        rlm.rlm_scan_prefill(p[..., :D], p[..., D:], s, state_out=self.state, saved=saved, lengths=lengths)
        out = torch.empty_like(h)
        rlm.rlm_linear(s, self.w_out, out, residual=h)
        self.kept = h, p, s, saved, lengths
        return out

    def backward(self, d_out: torch.Tensor) -> torch.Tensor:
        h, p, s, saved, lengths = self.kept
        D, g = self.D, self.grads
        ds, dp, dh = torch.empty_like(s), torch.empty_like(p), torch.empty_like(h)
        rlm.rlm_linear_backward(d_out, s, self.w_out, dx=ds, dw=g["w_out"])
        rlm.rlm_scan_backward(ds, p[..., :D], p[..., D:], saved, dp[..., :D], dp[..., D:], lengths=lengths)
        rlm.rlm_linear_backward(dp, h, self.w_in, dx=dh, dw=g["w_in"], dbias=g["b_in"])
        return dh.add_(d_out)                                                      # the residual's gradient

    def decode(self, h: torch.Tensor) -> torch.Tensor:
        """One token [B][D]; the state advances in place."""
        B, D = h.shape
        p, s, out = (torch.empty(B, n, dtype=BF16, device="cuda") for n in (2 * D, D, D))
        rlm.rlm_linear(h, self.w_in, p, bias=self.b_in)
        rlm.rlm_scan_decode(p[:, :D], p[:, D:], self.state, s)
        rlm.rlm_linear(s, self.w_out, out, residual=h)
        return out


class Model:
    def __init__(self, D: int, layers: int, bits: int = 32, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.blocks = [Block(D, gen) for _ in range(layers)]
        # bf16 matrices with fp32 masters, fp32 vectors: a group of each kind.
        mats = [(b, k) for b in self.blocks for k in ("w_in", "w_out")]
        weights = [getattr(b, k) for b, k in mats]
        self.groups = [
            rlm.AdamGroup(weights, [b.grads[k] for b, k in mats], [rlm.AdamState.zeros(w, bits) for w in weights],
                          [w.float() for w in weights]),
            rlm.AdamGroup([b.b_in for b in self.blocks], [b.grads["b_in"] for b in self.blocks],
                          [rlm.AdamState.zeros(b.b_in, bits) for b in self.blocks])]
        self.step = 0

    def forward(self, h, lengths=None):
        for b in self.blocks:
            h = b.forward(h, lengths)
        return h

    def train_step(self, u, target, lr):
        y = self.forward(u)
        diff = y.float() - target
        d = (2 / diff.numel() * diff).to(BF16)
        for b in reversed(self.blocks):
            d = b.backward(d)
        self.step += 1
        for g in self.groups:
            rlm.rlm_adamw_step(g, self.step, lr, beta2=0.99, weight_decay=0.01)
        return diff.square().mean()

    def decode(self, h):
        for b in self.blocks:
            h = b.decode(h)
        return h


def batch(B, L, D, gen):
    """Noise and its running averages: a_t = 0.9 a_{t-1} + 0.1 u_t."""
    u = torch.randn(B, L, D, generator=gen, device="cuda")
    k = 0.1 * 0.9 ** torch.arange(L - 1, -1, -1, device="cuda", dtype=torch.float32)
    pad = torch.nn.functional.pad(u.transpose(1, 2), (L - 1, 0)).reshape(B * D, 1, -1)
    a = torch.nn.functional.conv1d(pad, k.view(1, 1, -1)).view(B, D, L).transpose(1, 2)
    return u.to(BF16), a


def main(steps=200, bits=32, B=8, L=256, D=64, layers=2, quiet=False):
    """Trains, then decodes; returns the first and last losses and the decode's distance from the full pass."""
    model = Model(D, layers, bits)
    gen = torch.Generator(device="cuda").manual_seed(1)
    losses = []
    for i in range(steps):
        u, target = batch(B, L, D, gen)
        losses.append(model.train_step(u, target, 3e-3))
        if not quiet and i % 20 == 0:
            print(f"step {i:4d}  loss {losses[-1].item():.4f}")
    # Prompts of different lengths as one padded batch, then token by token.
    u, _ = batch(B, L, D, gen)
    T = 16
    lengths = torch.randint(1, L - T, (B,), generator=gen, device="cuda", dtype=torch.int32)
    full = model.forward(u)
    model.forward(u, lengths)
    worst = torch.zeros((), device="cuda")
    rows = torch.arange(B, device="cuda")
    for t in range(T):
        y = model.decode(u[rows, lengths.long() + t])
        worst = torch.maximum(worst, (y - full[rows, lengths.long() + t]).abs().max())
    first, last, worst = losses[0].item(), losses[-1].item(), worst.item()
    assert rlm.rlm_get_device_status() == rlm.RLM_OK
    if not quiet:
        print(f"loss {first:.4f} -> {last:.4f}; decoding differs from the full pass by at most {worst:.4f}")
    return first, last, worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args()
    main(a.steps, a.bits)
