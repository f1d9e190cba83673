"""Argument checks of the linear layer's C entry points (no GPU: nothing is enqueued)."""
import ctypes

import pytest

import paper_2607_05583_gb300 as rlm
from paper_2607_05583_gb300 import build as cbuild

FAKE, GB = 0x7F0000000000, 1 << 30
R, K, N = 100, 64, 128


@pytest.fixture(scope="module")
def lib():
    cbuild.build()
    return rlm.load_library()


def mat(k, rows, cols, ld=None, dt=rlm.RLM_BF16, off=0):
    return rlm._Matrix(FAKE + k * GB + off, dt, rows, cols, cols if ld is None else ld)


def ref(v):
    return None if v is None else ctypes.byref(v)


NO_LAUNCH = ctypes.POINTER(rlm._Launch)()


def forward(lib, x=mat(0, R, K), w=mat(1, N, K), bias=FAKE + 8 * GB, act=1, residual=mat(2, R, N), pre=mat(3, R, N),
            y=mat(4, R, N)):
    return lib.rlm_linear(ref(x), ref(w), bias, act, ref(residual), ref(pre), ref(y), NO_LAUNCH)


def backward(lib, dy=mat(0, R, N), x=mat(1, R, K), w=mat(2, N, K), pre=mat(3, R, N), act=1, dx=mat(4, R, K),
             dw=mat(5, N, K), dbias=FAKE + 8 * GB):
    return lib.rlm_linear_backward(ref(dy), ref(x), ref(w), ref(pre), act, ref(dx), ref(dw), dbias, NO_LAUNCH)


def test_good_arguments_reach_the_launch(lib):
    for kw in ({}, dict(residual=mat(4, R, N)), dict(residual=None, pre=None, bias=None, act=0)):
        assert forward(lib, **kw) == rlm.RLM_ERR_INVALID_ARG and b"launch is NULL" in lib.rlm_last_error()
    for kw in ({}, dict(dw=mat(5, N, K, dt=rlm.RLM_F32)), dict(dx=None, dw=None), dict(act=0, pre=None),
               dict(dy=mat(0, R, N, ld=256), x=mat(0, R, K, ld=256, off=256))):
        assert backward(lib, **kw) == rlm.RLM_ERR_INVALID_ARG and b"launch is NULL" in lib.rlm_last_error(), kw


INVALID = [dict(x=None), dict(w=None), dict(y=None), dict(x=mat(0, 0, K)), dict(x=mat(0, R, 60), w=mat(1, N, 60)),
           dict(w=mat(1, N, 72)), dict(w=mat(1, 12, K)), dict(y=mat(4, R, 120)), dict(y=mat(4, 99, N)),
           dict(x=mat(0, R, K, off=8)), dict(x=mat(0, R, K, ld=56)), dict(x=mat(0, R, K, ld=68)),
           dict(x=mat(0, R, K, dt=9)), dict(act=4), dict(act=-1), dict(bias=FAKE + 4), dict(y=mat(0, R, N)),
           dict(y=mat(1, R, N)), dict(pre=mat(4, R, N)), dict(residual=mat(4, R, N, off=256)),
           dict(residual=mat(3, R, N)), dict(bias=FAKE + 4 * GB), dict(residual=mat(2, R, 64))]


@pytest.mark.parametrize("k", range(len(INVALID)))
def test_forward_refusals(lib, k):
    assert forward(lib, **INVALID[k]) == rlm.RLM_ERR_INVALID_ARG
    assert b"launch" not in lib.rlm_last_error(), INVALID[k].keys()


INVALID_B = [dict(dy=None), dict(pre=None), dict(act=0), dict(dx=None, dw=None, dbias=None), dict(dy=mat(0, R, K)),
             dict(dx=mat(0, R, K)), dict(dw=mat(4, N, K)), dict(dbias=FAKE + 5 * GB), dict(dbias=FAKE + 2),
             dict(dx=mat(4, R, N)), dict(dw=mat(5, K, N)), dict(dx=mat(3, R, K))]


@pytest.mark.parametrize("k", range(len(INVALID_B)))
def test_backward_refusals(lib, k):
    assert backward(lib, **INVALID_B[k]) == rlm.RLM_ERR_INVALID_ARG
    assert b"launch" not in lib.rlm_last_error(), INVALID_B[k].keys()


def test_unsupported(lib):
    f32 = rlm.RLM_F32
    for kw in (dict(x=mat(0, R, K, dt=f32)), dict(w=mat(1, N, K, dt=f32)), dict(y=mat(4, R, N, dt=f32)),
               dict(x=mat(0, (1 << 24) + 1, K), y=mat(9, (1 << 24) + 1, N), residual=None, pre=None),
               dict(w=mat(1, (1 << 20) + 8, K), y=mat(9, R, (1 << 20) + 8), residual=None, pre=None)):
        assert forward(lib, **kw) == rlm.RLM_ERR_UNSUPPORTED
    assert backward(lib, dx=mat(4, R, K, dt=f32)) == rlm.RLM_ERR_UNSUPPORTED


def test_python_checks():
    import torch
    cpu = torch.zeros(8, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        rlm.rlm_linear(cpu, cpu, cpu)
    with pytest.raises(ValueError):
        rlm._act("relu")
