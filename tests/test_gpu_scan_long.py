"""Recurrences of many waves of tiles against the fp64 recurrence: the rings, the exchange's places and the
carries are used again and again.  Channels do not meet, so some of them are compared, all groups among them.

Tolerances as in test_gpu_scan: bf16 fields 2^-8, fp32 fields and states 2e-5 of the norm and 1e-4 of the largest."""
import numpy as np
import pytest

import _scan_ref as ref
from _util import rel_errors, to_np

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")

BOUND = {"bf16": (2.0 ** -8, 2.0 ** -8), "f32": (2e-5, 1e-4)}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# Segmented with narrow groups (10 waves), segmented with wide ones (the library's headline field: 32 waves in
# bf16), and enough chains that each CTA takes a row's 24 tiles alone.
SHAPES = [(1, 40000, 8), (4, 8192, 256), (4, 32768, 256), (24, 1500, 1024)]


def near(got, want, dtype, what):
    l2, mx = rel_errors(got, want)
    bl, bm = BOUND[dtype]
    assert l2 <= bl and mx <= bm, f"{what}: l2 {l2:.3e} > {bl} or max {mx:.3e} > {bm}"


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_many_waves(shape, dtype, ragged):
    B, L, D = shape
    leak = (B + ragged) % 2 == 0
    gen = torch.Generator(device="cuda").manual_seed(L + D)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, g, dy = randn(*shape).to(DT[dtype]), (2.5 + 1.5 * randn(*shape)).to(DT[dtype]), randn(*shape).to(DT[dtype])
    h0, dh = randn(B, D), randn(B, D)
    n = None
    if ragged:
        n = torch.randint(L // 2, L + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        n[0] = L - 3
        for t in (x, g, dy):
            t.masked_fill_((torch.arange(L, device="cuda")[None, :] >= n[:, None])[..., None], float("nan"))

    def run():
        y, dx, dg = (torch.full_like(x, 7.0) for _ in range(3))
        state, dh0 = torch.empty_like(h0), torch.empty_like(h0)
        saved = rlm.scan_saved(B, L, D)
        rlm.rlm_scan_prefill(x, g, y, leak=leak, state_in=h0, state_out=state, saved=saved, lengths=n)
        rlm.rlm_scan_backward(dy, x, g, saved, dx, dg, leak=leak, d_state_out=dh, d_state_in=dh0, lengths=n)
        return y, state, dx, dg, dh0

    got = run()
    assert rlm.rlm_get_device_status() == rlm.RLM_OK
    assert all(torch.equal(a, b) for a, b in zip(got, run()))
    at = torch.arange(D, device="cuda")[:: max(1, D // 29)]
    cut = lambda t: to_np(t[..., at])
    lengths = None if n is None else n.cpu().numpy()
    y, state, before = ref.forward(cut(x), cut(g), leak, cut(h0), lengths)
    dx, dg, dh0 = ref.backward(cut(dy), cut(x), cut(g), leak, before, cut(dh), lengths)
    for k, (want, kind) in enumerate(((y, dtype), (state, "f32"), (dx, dtype), (dg, dtype), (dh0, "f32"))):
        near(cut(got[k]), want, kind, ("y", "state", "dx", "dg", "d_state_in")[k])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,L,D", [(2, 700, 64), (3, 130, 24)])
def test_time_first_views(B, L, D, dtype):
    """All fields with time first, dx and dg as halves of one [L][B][2 D] buffer."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    f, dy = (torch.randn(L, B, n, generator=gen, device="cuda").to(DT[dtype]).transpose(0, 1) for n in (2 * D, D))
    x, g = f[..., :D], f[..., D:]
    out = []
    for first in (True, False):
        d = torch.empty(L, B, 2 * D, dtype=DT[dtype], device="cuda").transpose(0, 1)
        if not first:
            d, x, g, dy = (t.contiguous() for t in (d, x, g, dy))
        y, saved = torch.empty_like(x), rlm.scan_saved(B, L, D)
        rlm.rlm_scan_prefill(x, g, y, saved=saved)
        rlm.rlm_scan_backward(dy, x, g, saved, d[..., :D], d[..., D:])
        out.append((y, d))
    assert all(torch.equal(a, b) for a, b in zip(*out))
