"""Calls on a stream that is not the current one: where their workspace comes from, and what they cost the host."""
import time

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
rlm = pytest.importorskip("paper_2607_05583_gb300")


def prefill(stream):
    B, L, D, M = 2, 100, 64, 4
    x = torch.ones(B, L, D, dtype=torch.bfloat16, device="cuda")
    p = rlm.Params(*(torch.full((D, M), 0.5, device="cuda") for _ in range(4)))
    y = torch.empty_like(x)
    assert rlm.rlm_prefill_workspace_size(B, L, D, M, rlm.RLM_BF16) > 0
    return lambda: rlm.rlm_mix_prefill(x, p, y, stream=stream), y


@pytest.mark.parametrize("kind", ["stream", "handle", "legacy default"])
def test_workspaces_of_other_streams(kind):
    """The workspace comes from the call's stream's pool, and goes back to it."""
    side = torch.cuda.Stream()
    stream = {"stream": side, "handle": side.cuda_stream, "legacy default": 0}[kind]
    call, y = prefill(stream)
    want, ref = prefill(None)
    want()
    torch.cuda.synchronize()
    call()
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    for _ in range(200):
        call()
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == held
    assert torch.equal(y, ref)


def test_a_call_on_another_stream_costs_the_host_little_more():
    """The least of blocks of calls taken in turn: within 6 us of the call on the current stream."""
    calls = [prefill(None)[0], prefill(torch.cuda.Stream())[0]]
    times = [[], []]
    for rep in range(15):
        for call, ts in zip(calls, times):
            torch.cuda.synchronize()
            t = time.perf_counter()
            for _ in range(100):
                call()
            torch.cuda.synchronize()
            ts.append((time.perf_counter() - t) / 100 * 1e6)
    here, other = (min(ts) for ts in times)
    assert other <= here + 6, (here, other)
