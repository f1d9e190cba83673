"""Argument checks of the gated linear recurrence's C entry points (no GPU: nothing is enqueued)."""
import ctypes

import pytest

import paper_2607_05583_gb300 as rlm
from paper_2607_05583_gb300 import build as cbuild

FAKE = 0x7F0000000000
GB = 1 << 30


@pytest.fixture(scope="module")
def lib():
    cbuild.build()
    return rlm.load_library()


def field(k=0, B=2, L=100, D=64, dt=rlm.RLM_BF16, sb=None, sl=None, off=0):
    sl = D if sl is None else sl
    return rlm._Strided(FAKE + k * GB + off, dt, B, L, D, L * sl if sb is None else sb, sl)


def ref(v):
    return None if v is None else ctypes.byref(v)


def launch(nbytes=1 << 30):
    return ctypes.byref(rlm._Launch(None, FAKE + 30 * GB, nbytes))


def prefill(lib, x=None, g=None, y=None, sin=FAKE + 10 * GB, sout=FAKE + 11 * GB, saved=FAKE + 12 * GB, lengths=None,
            ln=None):
    f = lambda v, k: field(k) if v is None else v
    return lib.rlm_scan_prefill(ref(f(x, 0)), ref(f(g, 1)), 1, sin, ref(f(y, 2)), sout, saved, lengths,
                                launch() if ln is None else ln)


BAD = {
    "null pointer": dict(x=rlm._Strided(None, 1, 2, 100, 64, 6400, 64)),
    "misaligned": dict(x=field(0, off=8)),
    "dtype": dict(x=field(0, dt=7)),
    "no tokens": dict(x=field(0, L=0), g=field(1, L=0), y=field(2, L=0)),
    "odd width": dict(x=field(0, D=12), g=field(1, D=12), y=field(2, D=12)),
    "gate shape": dict(g=field(1, L=99)),
    "output dtype": dict(y=field(2, dt=rlm.RLM_F32)),
    "stride of 4 elements": dict(x=field(0, sl=68)),
    "negative stride": dict(x=field(0, sl=-64)),
    "rows overlap": dict(y=field(2, sl=32, sb=6400)),
    "batch rows overlap": dict(y=field(2, sb=64)),
    "output over input": dict(y=field(0, off=128)),
    "output over gate": dict(y=field(1)),
    "columns overlap": dict(x=field(0, sl=192), y=field(0, sl=192, off=64)),
    "state over field": dict(sout=FAKE + 2 * GB),
    "state misaligned": dict(sin=FAKE + 10 * GB + 4),
    "states overlap": dict(sin=FAKE + 10 * GB, sout=FAKE + 10 * GB + 256),
    "saved over state": dict(saved=FAKE + 11 * GB),
    "lengths misaligned": dict(lengths=FAKE + 2),
    "no launch": dict(ln=ctypes.POINTER(rlm._Launch)()),
}


@pytest.mark.parametrize("name", BAD)
def test_prefill_refusals(lib, name):
    assert prefill(lib, **BAD[name]) == rlm.RLM_ERR_INVALID_ARG, name
    assert lib.rlm_last_error()


def test_limits(lib):
    for kw in (dict(B=70000), dict(L=(1 << 24) + 1), dict(D=(1 << 20) + 8)):
        f = [field(k, **{**dict(B=1, L=1), **kw}) for k in (0, 40, 80)]
        assert prefill(lib, *f) == rlm.RLM_ERR_UNSUPPORTED


def backward(lib, dy=None, x=None, g=None, dx=None, dg=None, saved=FAKE + 12 * GB, dsin=FAKE + 13 * GB):
    f = lambda v, k: field(k) if v is None else v
    return lib.rlm_scan_backward(ref(f(dy, 0)), ref(f(x, 1)), ref(f(g, 2)), saved, 1, None, ref(f(dx, 3)),
                                 ref(f(dg, 4)), dsin, None, ctypes.POINTER(rlm._Launch)())


def test_backward_refusals(lib):
    bad = [dict(saved=None), dict(dx=field(1)), dict(dg=field(3)), dict(dy=field(0, B=3)), dict(dsin=FAKE + 12 * GB),
           dict(dg=field(4, dt=rlm.RLM_F32)), dict(dx=field(3, sl=0, sb=0))]
    for kw in bad:
        assert backward(lib, **kw) == rlm.RLM_ERR_INVALID_ARG, kw
    # Two halves of one buffer are apart: the call gets as far as its launch context.
    assert backward(lib, dx=field(3, sl=128), dg=field(3, sl=128, off=128)) == rlm.RLM_ERR_INVALID_ARG
    assert b"launch is NULL" in lib.rlm_last_error()


def test_decode_refusals(lib):
    def call(x, g, state, y):
        return lib.rlm_scan_decode(ref(x), ref(g), 0, state, ref(y), launch())
    f = lambda k, **kw: field(k, **{**dict(L=1), **kw})
    for args in ((field(0), field(1), FAKE + 10 * GB, field(2)), (f(0), f(1), None, f(2)), (f(0), f(1), FAKE, f(2)),
                 (f(0), f(1), FAKE + 10 * GB, f(2, sb=0)), (f(0), f(1), FAKE + 10 * GB, f(0)),
                 (None, f(1), FAKE + 10 * GB, f(2))):
        assert call(*args) == rlm.RLM_ERR_INVALID_ARG


def test_sizes(lib):
    assert rlm.rlm_scan_saved_size(2, 65, 8) == 2 * 2 * 8 * 4
    assert rlm.rlm_scan_saved_size(0, 65, 8) == 0


def test_strides_beyond_any_memory(lib):
    """Extents that would pass 64 bits (2^24 rows, 2^40 apart) are refused, not wrapped round."""
    L, sl = 1 << 24, 1 << 40
    far = field(0, B=1, L=L, sl=sl, sb=0)
    assert prefill(lib, far, field(1, B=1, L=L, sl=64), field(2, B=1, L=L, sl=64), ln=ctypes.POINTER(rlm._Launch)()) \
        == rlm.RLM_ERR_INVALID_ARG
    assert b"x has a stride" in lib.rlm_last_error()
