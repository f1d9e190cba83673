"""Argument checks of the optimizer step's C entry point (no GPU: nothing is enqueued)."""
import ctypes

import pytest

import paper_2607_05583_gb300 as rlm
from paper_2607_05583_gb300 import build as cbuild

FAKE, GB = 0x7F0000000000, 1 << 30


@pytest.fixture(scope="module")
def lib():
    cbuild.build()
    return rlm.load_library()


def entry(n=1000, **kw):
    v = dict(param=FAKE, grad=FAKE + GB, exp_avg=FAKE + 2 * GB, exp_avg_sq=FAKE + 3 * GB, exp_avg_scale=None,
             exp_avg_sq_scale=None, master=None, n=n)
    v.update(kw)
    return rlm._AdamTensor(**v)


def call(lib, entries, param=rlm.RLM_F32, grad=rlm.RLM_F32, bits=32, scale=None, count=None, **hyper):
    h = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=1)
    h.update(hyper)
    arr = (rlm._AdamTensor * max(1, len(entries)))(*entries)
    return lib.rlm_adamw_step(arr, len(entries) if count is None else count, param, grad, bits,
                              ctypes.byref(rlm._AdamHyper(**h)), scale, ctypes.POINTER(rlm._Launch)())


SCALES = dict(exp_avg_scale=FAKE + 5 * GB, exp_avg_sq_scale=FAKE + 6 * GB)


def test_good_arguments_reach_the_launch(lib):
    for kw in (dict(entries=[entry()]), dict(entries=[entry(**SCALES), entry(7, **SCALES)], bits=8),
               dict(entries=[entry(master=FAKE + 7 * GB)], param=rlm.RLM_BF16, grad=rlm.RLM_BF16),
               dict(entries=[entry(param=FAKE + 2)], param=rlm.RLM_BF16), dict(entries=[entry()], lr=0.0, beta1=0.0)):
        assert call(lib, **kw) == rlm.RLM_ERR_INVALID_ARG and b"launch is NULL" in lib.rlm_last_error(), kw


BAD = [dict(entries=[entry()], count=0), dict(entries=[entry(0)]), dict(entries=[entry(param=None)]),
       dict(entries=[entry(grad=None)]), dict(entries=[entry(exp_avg_sq=None)]), dict(entries=[entry(param=FAKE + 2)]),
       dict(entries=[entry(exp_avg=FAKE + 2 * GB + 1)]), dict(entries=[entry()], bits=8), dict(entries=[entry()], bits=16),
       dict(entries=[entry(**{**SCALES, "exp_avg_scale": FAKE + 5 * GB + 2})], bits=8),
       dict(entries=[entry(master=FAKE + 7 * GB)]),
       dict(entries=[entry(master=FAKE + 7 * GB), entry()], param=rlm.RLM_BF16),
       dict(entries=[entry(), entry(master=FAKE + 7 * GB)], param=rlm.RLM_BF16),
       dict(entries=[entry()], param=5), dict(entries=[entry()], grad=5), dict(entries=[entry()], scale=FAKE + 1),
       dict(entries=[entry(exp_avg=FAKE + GB + 512)]), dict(entries=[entry(grad=FAKE + 3996)])]
BAD += [dict(entries=[entry()], **{k: v}) for k, v in
        (("lr", -1.0), ("lr", float("nan")), ("eps", float("inf")), ("weight_decay", -0.1), ("beta1", 1.0),
         ("beta2", float("nan")), ("beta2", -0.1), ("step", 0))]


@pytest.mark.parametrize("k", range(len(BAD)))
def test_refusals(lib, k):
    assert call(lib, **BAD[k]) == rlm.RLM_ERR_INVALID_ARG
    assert b"launch" not in lib.rlm_last_error(), BAD[k]


def test_unsupported(lib):
    assert call(lib, [entry((1 << 40) + 1)]) == rlm.RLM_ERR_UNSUPPORTED
