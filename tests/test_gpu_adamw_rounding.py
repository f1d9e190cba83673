"""8-bit moments over many steps: they move as the 32-bit ones do, although a step's change is a small part
of the distance between two codes.

Tolerances.  A code's distance is 1/16 to 1/8 of its value, a step's error at most that, independent from
step to step and without a mean: at beta2 = 0.95, an error of 0.035 a step remembered for about 40 steps, half
of them in effect, gives 0.035 sqrt(20) = 0.16 of a value, at beta2 = 0.999 the same (a smaller error, remembered
longer).  The mean over 4096 values is then within 0.16 / 64 = 0.3 %, and the root of a square with that spread
has a mean off by 0.16^2 / 2 = 1.3 %: 4 % holds both, and the steps whose change is rounded to nearest."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")

BETAS = [(0.9, 0.95), (0.9, 0.999), (0.95, 0.99), (0.99, 0.999)]
N = 4096


class Pair:
    """The same weights and gradients, moments in 8 and in 32 bits."""

    def __init__(self, n=N, seed=0):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        p = self.randn(n)
        self.g = torch.zeros_like(p)
        self.p = [p.clone(), p.clone()]
        self.st = [rlm.AdamState.zeros(p, bits) for bits in (8, 32)]
        self.group = [rlm.AdamGroup([w], [self.g], [s]) for w, s in zip(self.p, self.st)]
        self.t = 0

    def randn(self, n=N):
        return torch.randn(n, generator=self.gen, device="cuda")

    def steps(self, n, grad, betas, lr=1e-3):
        for _ in range(n):
            self.t += 1
            self.g.copy_(grad())
            for group in self.group:
                rlm.rlm_adamw_step(group, self.t, lr, beta1=betas[0], beta2=betas[1], weight_decay=0.0)

    def roots(self):
        """sqrt(v) of both."""
        return [s.values()[1].double().sqrt() for s in self.st]

    def ms(self):
        return [s.values()[0].double() for s in self.st]


def slope(a, b):
    return (a @ b / (b @ b)).item()


@pytest.mark.parametrize("betas", BETAS)
def test_random_gradients(betas):
    """The second moment settles where the 32-bit one does, and follows gradients that fall tenfold."""
    pair = Pair()
    pair.steps(600, pair.randn, betas)
    a, b = pair.roots()
    assert abs((a / b).mean().item() - 1) < 0.04
    assert abs(slope(*pair.ms()) - 1) < 0.04
    pair.steps(600, lambda: 0.1 * pair.randn(), betas)
    a, b = pair.roots()
    assert abs((a / b).mean().item() - 1) < 0.05         # (a spread that is still that of the larger gradients)


@pytest.mark.parametrize("betas", BETAS)
def test_constant_gradients(betas):
    """m and sqrt(v) arrive at the gradient, and the weights go the same way."""
    pair = Pair(seed=1)
    g = pair.randn()
    pair.steps(1000, lambda: g, betas)
    a, b = pair.roots()
    big = g.abs() > 0.05                                # (below, sqrt(v) meets its smallest code)
    assert abs((a / b)[big].mean().item() - 1) < 0.04
    assert abs(slope(*pair.ms()) - 1) < 0.02
    start = [p.clone() for p in pair.p]
    pair.steps(100, lambda: g, betas)
    moved = [(p - s).double()[big] for p, s in zip(pair.p, start)]
    assert abs(slope(*moved) - 1) < 0.04


@pytest.mark.parametrize("betas", BETAS)
def test_no_gradients(betas):
    """Both moments decay: half-lives of 14 to 1400 steps.  With no gradients nothing pulls a value back, so its
    errors add up as a random walk: 300 steps of 0.035 are 0.6 of a value and 1 % of the mean."""
    pair = Pair(seed=2)
    pair.steps(200, pair.randn, betas)
    zero = torch.zeros_like(pair.g)
    m0 = pair.ms()[1].abs().sum()
    pair.steps(300, lambda: zero, betas)
    a, b = pair.roots()
    assert abs((a.sum() / b.sum()).item() - 1) < 0.06
    assert pair.ms()[0].abs().sum() < 3 * pair.ms()[1].abs().sum() + 1e-4 * m0
    pair.steps(700, lambda: zero, betas)
    a, b = pair.roots()
    assert abs(np.log((a.sum() / b.sum()).item())) < 0.3


@pytest.mark.parametrize("betas", [(0.99, 0.999), (0.95, 0.95)])
def test_small_gradients_beside_large_ones(betas):
    """Values 2^11 to 2^13 below their block's largest: a step's (1 - beta1) g alone is below the smallest code."""
    pair = Pair(seed=3)
    g = torch.where(torch.arange(N, device="cuda") % 256 == 0, 1.0, 2.0 ** -11 * (0.25 + 0.75 * torch.rand(N, device="cuda")))
    pair.steps(1500, lambda: g, betas)
    small = g < 0.5
    a, b = (m[small] for m in pair.ms())
    assert abs((a.sum() / b.sum()).item() - 1) < 0.05


def test_rounding_is_reproducible_and_changes_with_the_step():
    def codes(steps, sizes=(700, 256, 1), seed=4):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        ps = [torch.randn(n, generator=gen, device="cuda") for n in sizes]
        gs = [torch.randn(n, generator=gen, device="cuda") for n in sizes]
        sts = [rlm.AdamState.zeros(p, 8) for p in ps]
        group = rlm.AdamGroup(ps, gs, sts)
        for t in steps:
            rlm.rlm_adamw_step(group, t, 1e-3, beta2=0.999)
        return torch.cat([torch.cat([s.m.view(torch.uint8), s.v.view(torch.uint8)]) for s in sts])

    base = codes(range(1, 50))
    assert torch.equal(base, codes(range(1, 50)))
    other = (base != codes(list(range(1, 49)) + [1000])).float().mean().item()
    assert 0 < other < 0.2


def test_gradients_that_are_not_finite():
    """NaN stays in its value, and an infinity leaves its value's moments infinite (and its block's scale large)."""
    pair = Pair(n=512, seed=5)
    g = pair.randn(512)
    g[7], g[300], g[301] = float("nan"), float("inf"), float("-inf")
    pair.steps(3, lambda: g, (0.9, 0.95))
    for s in pair.st:
        m, v = s.values()
        assert torch.isnan(m[7]) and torch.isnan(v[7])
        assert torch.isfinite(m[:256]).sum() == 255 and torch.isfinite(v[:256]).sum() == 255
        assert torch.isinf(m[300:302]).all() and torch.isinf(v[300:302]).all()


def test_states_of_a_group_share_their_rounding():
    p, q = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    a, b = rlm.AdamState.zeros(p, 8), rlm.AdamState.zeros(q, 8)
    assert a.draw and not rlm.AdamState.zeros(p, 32).draw
    b.draw = False
    with pytest.raises(ValueError):
        rlm.AdamGroup([p, q], [p.clone(), q.clone()], [a, b])


def test_nearest_codes_of_a_step():
    """To nearest, a step's codes are within half a code of its moments: 2^-4 of them in the normal range."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    p, g = (torch.randn(2048, generator=gen, device="cuda") for _ in range(2))
    a = rlm.AdamState.zeros(p, 8)
    rlm.rlm_adamw_step(rlm.AdamGroup([p], [g], [a]), 1, 1e-3)
    near = rlm.AdamState(*(t.clone() for t in (a.m, a.v, a.m_scale, a.v_scale)))
    m, v = (t.double() for t in near.values())
    rlm.rlm_adamw_step(rlm.AdamGroup([p], [g], [near]), 2, 1e-3, beta1=0.9, beta2=0.999)
    want = 0.9 * m + 0.1 * g.double(), (0.999 * v + 0.001 * g.double() ** 2).sqrt()
    for got, w, scale in zip((near.m, near.v), want, (near.m_scale, near.v_scale)):
        s = scale.double().repeat_interleave(256)
        off, normal = (got.double() * s - w).abs(), w.abs() > 2.0 ** -6 * s
        assert (off <= w.abs() * 2.0 ** -4 * 1.0001)[normal].all()
