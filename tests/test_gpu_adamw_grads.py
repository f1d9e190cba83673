"""AdamGroup over weights whose .grad it was given: a .grad that is no longer that buffer is an error, not a step
on old gradients."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")


def weights():
    ws = [torch.nn.Parameter(torch.ones(n, device="cuda")) for n in (300, 17)]
    for w in ws:
        w.grad = torch.full_like(w, 0.5)
    return ws


def group_of(ws):
    return rlm.AdamGroup(ws, [w.grad for w in ws], [rlm.AdamState.zeros(w) for w in ws])


def test_gradients_in_place_are_stepped_on():
    ws = weights()
    group = group_of(ws)
    for t in (1, 2):
        for w in ws:
            w.grad.zero_()
        sum((w * w).sum() for w in ws).backward()           # accumulates into the same buffers
        old = [w.detach().clone() for w in ws]
        rlm.rlm_adamw_step(group, t, 0.1, weight_decay=0.0)
        assert all((w < o).all() for w, o in zip(ws, old))


@pytest.mark.parametrize("how", ["set to none", "replaced", "one of them"])
def test_replaced_gradients_are_refused(how):
    ws = weights()
    group = group_of(ws)
    old = [w.detach().clone() for w in ws]
    for w in ws[1:] if how == "one of them" else ws:
        w.grad = None
    if how != "set to none":
        sum((w * w).sum() for w in ws).backward()
    with pytest.raises(ValueError, match="tensor [01].*grad"):
        rlm.rlm_adamw_step(group, 1, 0.1)
    torch.cuda.synchronize()
    assert all(torch.equal(w, o) for w, o in zip(ws, old))


def test_buffers_of_the_callers_own_are_not_looked_at():
    ws = weights()
    own = [torch.full_like(w, 0.25).detach() for w in ws]
    group = rlm.AdamGroup(ws, own, [rlm.AdamState.zeros(w) for w in ws])
    for w in ws:
        w.grad = None
    rlm.rlm_adamw_step(group, 1, 0.1, weight_decay=0.0)
    torch.cuda.synchronize()
    assert all((w < 1).all() for w in ws)
