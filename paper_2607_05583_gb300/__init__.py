"""Python binding of the GB300 causal resonant field mixing library (``librlm.so``).

Argument marshalling only: every step of the operator runs in the library's
CUDA kernels, reached through the C ABI declared in ``include/rlm.h`` with the
same function names.  PyTorch supplies device memory and the current stream.
There is no fallback: if the compiled library is missing the calls raise.

Names follow the paper (ResonatorLM, arxiv 2607.05583): x is the drive field
[B][L][D]; decay gamma, frequency omega, amplitude A and phase phi are the
per-mode resonator parameters [D][M]; the state is the complex recurrent state
of Sec. 3.3, [B][D][M] complex fp32 plus its mode coefficients.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

from . import build as _build_mod

__all__ = [
    "RlmError", "Params", "Grads", "State", "load_library", "library_path",
    "rlm_mix_prefill", "rlm_mix_prefill_from", "rlm_mix_prefill_noalloc", "rlm_mix_decode", "rlm_mix_backward",
    "rlm_mix_backward_from", "rlm_state_init", "Local", "ConvState", "Coupling", "rlm_mixer_prefill",
    "rlm_mixer_decode",
    "rlm_prefill_workspace_size", "rlm_backward_workspace_size",
    "rlm_scan_prefill", "rlm_scan_backward", "rlm_scan_decode", "rlm_scan_saved_size", "scan_saved",
    "rlm_linear", "rlm_linear_backward", "rlm_linear_workspace_size", "rlm_linear_backward_workspace_size",
    "AdamState", "AdamGroup", "rlm_adamw_step",
    "rlm_validate_params", "rlm_get_device_status", "rlm_status_string",
    "rlm_version", "rlm_kernels_launched", "RLM_OK", "RLM_ERR_INVALID_ARG", "RLM_ERR_UNSUPPORTED",
    "RLM_ERR_CUDA", "RLM_ERR_TIMEOUT", "RLM_F32", "RLM_BF16",
]

RLM_OK, RLM_ERR_INVALID_ARG, RLM_ERR_UNSUPPORTED, RLM_ERR_CUDA, RLM_ERR_TIMEOUT = range(5)
RLM_F32, RLM_BF16 = 0, 1


class _Tensor(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("dtype", ctypes.c_int),
                ("B", ctypes.c_int64), ("L", ctypes.c_int64), ("D", ctypes.c_int64)]


class _Params(ctypes.Structure):
    _fields_ = [("decay", ctypes.c_void_p), ("freq", ctypes.c_void_p),
                ("amp", ctypes.c_void_p), ("phase", ctypes.c_void_p),
                ("D", ctypes.c_int), ("M", ctypes.c_int)]


_Grads = _Params


class _State(ctypes.Structure):
    _fields_ = [("s", ctypes.c_void_p), ("coef", ctypes.c_void_p),
                ("B", ctypes.c_int), ("D", ctypes.c_int), ("M", ctypes.c_int)]


class _Local(ctypes.Structure):
    _fields_ = [("conv_w", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("D", ctypes.c_int), ("K", ctypes.c_int)]


class _Coupling(ctypes.Structure):
    _fields_ = [("c_raw", ctypes.c_void_p), ("lambda_c", ctypes.c_float), ("H", ctypes.c_int)]


class _ConvState(ctypes.Structure):
    _fields_ = [("u", ctypes.c_void_p), ("dtype", ctypes.c_int), ("B", ctypes.c_int64),
                ("D", ctypes.c_int), ("K", ctypes.c_int)]


class _Strided(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("dtype", ctypes.c_int),
                ("B", ctypes.c_int64), ("L", ctypes.c_int64), ("D", ctypes.c_int64),
                ("stride_b", ctypes.c_int64), ("stride_l", ctypes.c_int64)]


class _Matrix(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("dtype", ctypes.c_int),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64)]


class _AdamTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("exp_avg", ctypes.c_void_p),
                ("exp_avg_sq", ctypes.c_void_p), ("exp_avg_scale", ctypes.c_void_p),
                ("exp_avg_sq_scale", ctypes.c_void_p), ("master", ctypes.c_void_p), ("n", ctypes.c_int64)]


class _AdamHyper(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("step", ctypes.c_int64)]


class _Launch(ctypes.Structure):
    _fields_ = [("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class RlmError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: {rlm_status_string(status)}: {detail}")
        self.status = status


_lib = None


def library_path() -> str:
    return _build_mod.LIB


def load_library(build_if_missing: bool = False) -> ctypes.CDLL:
    """Load librlm.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build_mod.LIB
    if not os.path.exists(path):
        if not build_if_missing:
            raise RuntimeError(
                f"the CUDA library {path} is not built; run "
                "`python -c 'import __graft_entry__ as g; g.build()'` first")
        _build_mod.build()
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    lib.rlm_mix_prefill.argtypes = [P(_Tensor), P(_Params), P(_Tensor), P(_State), P(_Launch)]
    lib.rlm_mix_prefill_from.argtypes = [P(_Tensor), P(_Params), P(_State), P(_Tensor), P(_State),
                                         P(_Launch)]
    lib.rlm_mix_decode.argtypes = [P(_Tensor), P(_State), P(_Tensor), P(_Launch)]
    lib.rlm_mix_backward.argtypes = [P(_Tensor), P(_Tensor), P(_Params), P(_Tensor),
                                     P(_Grads), P(_Launch)]
    lib.rlm_mix_backward_from.argtypes = [P(_Tensor), P(_Tensor), P(_Params), P(_State), P(_State),
                                          P(_Tensor), P(_Grads), P(_State), P(_Launch)]
    lib.rlm_mixer_prefill.argtypes = [P(_Tensor), P(_Tensor), P(_Params), P(_Local), P(_Coupling), P(_State),
                                      P(_ConvState), P(_Tensor), P(_State), P(_ConvState), P(_Launch)]
    lib.rlm_mixer_decode.argtypes = [P(_Tensor), P(_Tensor), P(_State), P(_Local), P(_Coupling), P(_ConvState),
                                     P(_Tensor), P(_Launch)]
    lib.rlm_state_init.argtypes = [P(_State), P(_Params), P(_Launch)]
    lib.rlm_validate_params.argtypes = [P(_Params)]
    lib.rlm_get_device_status.argtypes = [P(_Launch)]
    lib.rlm_test_stall_segments.argtypes = [ctypes.c_int]
    for f in ("rlm_prefill_workspace_size", "rlm_backward_workspace_size"):
        getattr(lib, f).argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int,
                                    ctypes.c_int, ctypes.c_int]
        getattr(lib, f).restype = ctypes.c_size_t
    for f in ("rlm_mix_prefill", "rlm_mix_prefill_from", "rlm_mix_decode", "rlm_mix_backward",
              "rlm_mix_backward_from", "rlm_mixer_prefill", "rlm_mixer_decode", "rlm_state_init",
              "rlm_validate_params", "rlm_get_device_status"):
        getattr(lib, f).restype = ctypes.c_int
    lib.rlm_status_string.argtypes = [ctypes.c_int]
    lib.rlm_status_string.restype = ctypes.c_char_p
    lib.rlm_last_error.restype = ctypes.c_char_p
    lib.rlm_version.restype = ctypes.c_int
    lib.rlm_kernels_launched.restype = ctypes.c_ulonglong
    lib.rlm_mix_prefill_noalloc.argtypes = [P(_Tensor), P(_Params), P(_Tensor), P(_State),
                                            ctypes.c_void_p]
    lib.rlm_mix_prefill_noalloc.restype = ctypes.c_int
    F, V, I = P(_Strided), ctypes.c_void_p, ctypes.c_int
    lib.rlm_scan_prefill.argtypes = [F, F, I, V, F, V, V, V, P(_Launch)]
    lib.rlm_scan_backward.argtypes = [F, F, F, V, I, V, F, F, V, V, P(_Launch)]
    lib.rlm_scan_decode.argtypes = [F, F, I, V, F, P(_Launch)]
    for f in ("rlm_scan_prefill", "rlm_scan_backward", "rlm_scan_decode"):
        getattr(lib, f).restype = ctypes.c_int
    lib.rlm_scan_saved_size.argtypes = [ctypes.c_int64, ctypes.c_int64, I]
    lib.rlm_scan_saved_size.restype = ctypes.c_size_t
    X, Q = P(_Matrix), ctypes.c_int64
    lib.rlm_linear.argtypes = [X, X, V, I, X, X, X, P(_Launch)]
    lib.rlm_linear_backward.argtypes = [X, X, X, X, I, X, X, V, P(_Launch)]
    lib.rlm_linear_workspace_size.argtypes = [Q, Q, Q]
    lib.rlm_linear_backward_workspace_size.argtypes = [Q, Q, Q, I]
    lib.rlm_adamw_step.argtypes = [P(_AdamTensor), I, I, I, I, P(_AdamHyper), V, P(_Launch)]
    for f in ("rlm_linear", "rlm_linear_backward", "rlm_adamw_step"):
        getattr(lib, f).restype = ctypes.c_int
    for f in ("rlm_linear_workspace_size", "rlm_linear_backward_workspace_size"):
        getattr(lib, f).restype = ctypes.c_size_t
    _lib = lib
    return lib


# --------------------------------------------------------------- containers
@dataclass
class Params:
    """Resonator parameters, each a float32 CUDA tensor [D][M]."""
    decay: torch.Tensor
    freq: torch.Tensor
    amp: torch.Tensor
    phase: torch.Tensor

    @property
    def D(self) -> int:
        return int(self.decay.shape[0])

    @property
    def M(self) -> int:
        return int(self.decay.shape[1])

    @classmethod
    def from_arrays(cls, decay, freq, amp, phase, device="cuda"):
        t = lambda a: torch.as_tensor(a, dtype=torch.float32).contiguous().to(device)
        return cls(t(decay), t(freq), t(amp), t(phase))

    @classmethod
    def tied_heads(cls, decay, freq, phase, d_h: int, device="cuda"):
        """The paper's parameterisation (Sec. 3.1): one damped mode per head, no
        amplitude (A = 1), shared by the head's d_h channels (head-major).  decay,
        freq, phase: [H].  Gives [H * d_h][1] parameters, which the bf16 prefill
        runs on its tcgen05 path (M = 1)."""
        t = lambda a: torch.as_tensor(a, dtype=torch.float32).reshape(-1).repeat_interleave(d_h)
        dec, fr, ph = t(decay), t(freq), t(phase)
        amp = torch.ones_like(dec)
        return cls(*(v.reshape(-1, 1).contiguous().to(device) for v in (dec, fr, amp, ph)))

    def _c(self) -> _Params:
        return _Params(*(_ptr(t, torch.float32, 2) for t in
                         (self.decay, self.freq, self.amp, self.phase)), self.D, self.M)


@dataclass
class Grads(Params):
    """Parameter gradients, same layout as Params (overwritten by backward)."""

    @classmethod
    def empty(cls, D: int, M: int, device="cuda"):
        return cls(*(torch.empty(D, M, dtype=torch.float32, device=device) for _ in range(4)))


@dataclass
class State:
    """Recurrent state of Sec. 3.3: s [B][D][M][2] (Re, Im) and coef [D][M][4]."""
    s: torch.Tensor
    coef: torch.Tensor

    @classmethod
    def empty(cls, B: int, D: int, M: int, device="cuda"):
        return cls(torch.empty(B, D, M, 2, dtype=torch.float32, device=device),
                   torch.empty(D, M, 4, dtype=torch.float32, device=device))

    @property
    def shape(self):
        B, D, M, _ = self.s.shape
        return int(B), int(D), int(M)

    def complex(self) -> torch.Tensor:
        return torch.view_as_complex(self.s.contiguous())

    def _c(self) -> _State:
        B, D, M = self.shape
        return _State(_ptr(self.s, torch.float32, 4), _ptr(self.coef, torch.float32, 3), B, D, M)


@dataclass
class Local:
    """Local lexical path of Sec. 3.4: depthwise causal kernel conv_w [D][K] (conv_w[d][k]
    multiplies u_{t-k}) and channel scale [D], both float32 CUDA tensors."""
    conv_w: torch.Tensor
    scale: torch.Tensor

    @property
    def K(self) -> int:
        return int(self.conv_w.shape[1])

    @classmethod
    def from_arrays(cls, conv_w, scale, device="cuda"):
        t = lambda a: torch.as_tensor(a, dtype=torch.float32).contiguous().to(device)
        return cls(t(conv_w), t(scale))

    def _c(self) -> _Local:
        D, K = self.conv_w.shape
        if K == 0:
            return _Local(None, None, int(D), 0)
        return _Local(_ptr(self.conv_w, torch.float32, 2), _ptr(self.scale, torch.float32, 1), int(D), int(K))


@dataclass
class Coupling:
    """Head coupling of Sec. 3.4: raw matrix c_raw [H][H] (float32 CUDA tensor) and
    strength lambda_c; C = I + lambda_c / sqrt(H) tanh(c_raw) mixes the heads of
    head-major channels."""
    c_raw: torch.Tensor
    lambda_c: float

    @classmethod
    def from_arrays(cls, c_raw, lambda_c, device="cuda"):
        return cls(torch.as_tensor(c_raw, dtype=torch.float32).contiguous().to(device), float(lambda_c))

    def _c(self) -> _Coupling:
        H = int(self.c_raw.shape[0])
        return _Coupling(_ptr(self.c_raw, torch.float32, 2), float(self.lambda_c), H)


@dataclass
class ConvState:
    """Drive history of the local path: u [B][K-1][D] in the field's dtype, oldest first."""
    u: torch.Tensor

    @property
    def K(self) -> int:
        return int(self.u.shape[1]) + 1

    @classmethod
    def empty(cls, B: int, D: int, K: int, dtype=torch.bfloat16, device="cuda"):
        return cls(torch.empty(B, max(K - 1, 0), D, dtype=dtype, device=device))

    def _c(self) -> _ConvState:
        if self.u.dtype not in _DT or not self.u.is_cuda or not self.u.is_contiguous() or self.u.dim() != 3:
            raise ValueError("ConvState.u must be a contiguous CUDA [B][K-1][D] float32 or bfloat16 tensor")
        B, K1, D = self.u.shape
        return _ConvState(self.u.data_ptr() if K1 > 0 else None, _DT[self.u.dtype], int(B), int(D), int(K1) + 1)


# --------------------------------------------------------------- marshalling
_DT = {torch.float32: RLM_F32, torch.bfloat16: RLM_BF16}


def _ptr(t: torch.Tensor, dtype, ndim) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch.Tensor")
    if t.dtype != dtype or t.dim() != ndim or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"expected a contiguous CUDA {dtype} tensor of rank {ndim}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _field(t: torch.Tensor) -> _Tensor:
    if t.dtype not in _DT:
        raise ValueError(f"unsupported dtype {t.dtype}")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("fields must be contiguous CUDA tensors")
    if t.dim() == 3:
        B, L, D = t.shape
    elif t.dim() == 2:     # a single token per batch row: [B][D]
        (B, D), L = t.shape, 1
    else:
        raise ValueError(f"fields are [B][L][D] (or [B][D] for one token), got {tuple(t.shape)}")
    return _Tensor(t.data_ptr(), _DT[t.dtype], B, L, D)


def _strided(t: torch.Tensor, name: str) -> _Strided:
    """A [B][L][D] (or, for one token, [B][D]) field, possibly a view with row strides."""
    dt, shape, st = _DT.get(t.dtype), t.shape, t.stride()
    if dt is None:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    if not t.is_cuda or len(shape) not in (2, 3) or st[-1] != 1:
        raise ValueError(f"{name} must be a CUDA [B][L][D] (or [B][D]) tensor with unit channel stride, got "
                         f"{tuple(shape)} with strides {st} on {t.device}")
    if len(shape) == 2:
        return _Strided(t.data_ptr(), dt, shape[0], 1, shape[1], st[0], shape[1])
    return _Strided(t.data_ptr(), dt, *shape, st[0], st[1])


def _matrix(t: torch.Tensor, name: str) -> _Matrix:
    """A row-major matrix [...][cols] whose leading dimensions share one row pitch."""
    dt, shape, st = _DT.get(t.dtype), t.shape, t.stride()
    if dt is None:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    if not t.is_cuda or len(shape) < 2 or st[-1] != 1:
        raise ValueError(f"{name} must be a CUDA matrix [...][cols] with unit column stride, got {tuple(shape)} with "
                         f"strides {st} on {t.device}")
    if len(shape) > 2:
        t = t.view(-1, shape[-1])          # raises where the rows do not share one pitch
        shape, st = t.shape, t.stride()
    rows, cols = shape
    return _Matrix(t.data_ptr(), dt, rows, cols, st[0] if rows > 1 else cols)


def _opt(t: torch.Tensor | None, dtype, shape, name: str):
    """Pointer of an optional contiguous CUDA tensor of a fixed shape (None: NULL)."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name} must be a contiguous CUDA {dtype} tensor of shape {tuple(shape)}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _launch(stream, workspace) -> _Launch:
    if workspace is None:
        return _Launch(_stream(stream), None, 0)
    return _Launch(_stream(stream), workspace.data_ptr(),
                   workspace.numel() * workspace.element_size())


def _check(status: int, where: str):
    if status != RLM_OK:
        raise RlmError(status, where, load_library().rlm_last_error().decode())


class _StreamMemory:
    """Bytes from the caching allocator's pool of a stream that need not be the current one."""

    def __init__(self, nbytes: int, device, stream: int):
        self._n = nbytes
        self._ptr = torch.cuda.caching_allocator_alloc(nbytes, device, stream)

    def data_ptr(self) -> int:
        return self._ptr

    def numel(self) -> int:
        return self._n

    def element_size(self) -> int:
        return 1

    def __del__(self):
        if self.__dict__.get("_ptr"):
            torch.cuda.caching_allocator_delete(self._ptr)


def _workspace(nbytes: int, device, stream=None):
    """A call's own workspace, from the allocator's pool of the stream that the call runs on: once
    released it goes to that stream's later work only."""
    if nbytes == 0:
        return None
    if stream is not None and (handle := _stream(stream)) != _stream(None):
        return _StreamMemory(nbytes, device, handle)
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


# --------------------------------------------------------------- entry points
def rlm_status_string(status: int) -> str:
    return load_library().rlm_status_string(status).decode()


def rlm_version() -> int:
    return load_library().rlm_version()


def rlm_kernels_launched() -> int:
    """Kernels the library has launched in this process (host-side count)."""
    return int(load_library().rlm_kernels_launched())


def rlm_prefill_workspace_size(B: int, L: int, D: int, M: int, dtype) -> int:
    return load_library().rlm_prefill_workspace_size(B, L, D, M, _DT.get(dtype, dtype))


def rlm_backward_workspace_size(B: int, L: int, D: int, M: int, dtype) -> int:
    return load_library().rlm_backward_workspace_size(B, L, D, M, _DT.get(dtype, dtype))


def rlm_mix_prefill(x: torch.Tensor, params: Params, y: torch.Tensor,
                    state_out: State | None = None, workspace: torch.Tensor | None = None,
                    stream=None) -> None:
    """Causal mixing y = K * x (Eq. 2) from a zero state; optional terminal state.

    ``workspace`` defaults to a fresh buffer of rlm_prefill_workspace_size bytes."""
    lib = load_library()
    xt, yt = _field(x), _field(y)
    if workspace is None:
        workspace = _workspace(lib.rlm_prefill_workspace_size(xt.B, xt.L, xt.D, params.M, xt.dtype),
                               x.device, stream)
    st = state_out._c() if state_out is not None else None
    _check(lib.rlm_mix_prefill(ctypes.byref(xt), ctypes.byref(params._c()), ctypes.byref(yt),
                               ctypes.byref(st) if st is not None else None,
                               ctypes.byref(_launch(stream, workspace))), "rlm_mix_prefill")


def rlm_mix_prefill_from(x: torch.Tensor, params: Params, state_in: State | None, y: torch.Tensor,
                         state_out: State | None = None, workspace: torch.Tensor | None = None,
                         stream=None) -> None:
    """Causal mixing from an initial state (chunked or continued prefill): y = K * x
    plus the free response of ``state_in`` (its ``s``; None = zero state).
    ``state_out`` may be ``state_in`` itself (in-place continuation)."""
    lib = load_library()
    xt, yt = _field(x), _field(y)
    if workspace is None:
        workspace = _workspace(lib.rlm_prefill_workspace_size(xt.B, xt.L, xt.D, params.M, xt.dtype),
                               x.device, stream)
    si = state_in._c() if state_in is not None else None
    so = state_out._c() if state_out is not None else None
    _check(lib.rlm_mix_prefill_from(ctypes.byref(xt), ctypes.byref(params._c()),
                                    ctypes.byref(si) if si is not None else None, ctypes.byref(yt),
                                    ctypes.byref(so) if so is not None else None,
                                    ctypes.byref(_launch(stream, workspace))), "rlm_mix_prefill_from")


def rlm_mix_prefill_noalloc(x: torch.Tensor, params: Params, y: torch.Tensor,
                            state_out: State | None = None, stream=None) -> None:
    """rlm_mix_prefill without a workspace, for callers that cannot allocate device
    memory: the scratch is the library's fixed 64 MiB device array (see rlm.h).
    Calls that overlap on the GPU race on that array."""
    lib = load_library()
    xt, yt = _field(x), _field(y)
    st = state_out._c() if state_out is not None else None
    _check(lib.rlm_mix_prefill_noalloc(ctypes.byref(xt), ctypes.byref(params._c()),
                                       ctypes.byref(yt),
                                       ctypes.byref(st) if st is not None else None,
                                       _stream(stream)), "rlm_mix_prefill_noalloc")


def rlm_mix_decode(x_t: torch.Tensor, state: State, y_t: torch.Tensor, stream=None) -> None:
    """One decode step (Eq. 4-5); the state is updated in place."""
    lib = load_library()
    xt, yt = _field(x_t), _field(y_t)
    _check(lib.rlm_mix_decode(ctypes.byref(xt), ctypes.byref(state._c()), ctypes.byref(yt),
                              ctypes.byref(_launch(stream, None))), "rlm_mix_decode")


def rlm_state_init(state: State, params: Params, stream=None) -> None:
    lib = load_library()
    _check(lib.rlm_state_init(ctypes.byref(state._c()), ctypes.byref(params._c()),
                              ctypes.byref(_launch(stream, None))), "rlm_state_init")


def rlm_mix_backward(dy: torch.Tensor, x: torch.Tensor, params: Params, dx: torch.Tensor,
                     dparams: Grads, workspace: torch.Tensor | None = None, stream=None) -> None:
    """dx and the four parameter gradients of l given dy = dl/dy."""
    lib = load_library()
    dyt, xt, dxt = _field(dy), _field(x), _field(dx)
    if workspace is None:
        workspace = _workspace(lib.rlm_backward_workspace_size(xt.B, xt.L, xt.D, params.M,
                                                               xt.dtype), x.device, stream)
    _check(lib.rlm_mix_backward(ctypes.byref(dyt), ctypes.byref(xt), ctypes.byref(params._c()),
                                ctypes.byref(dxt), ctypes.byref(dparams._c()),
                                ctypes.byref(_launch(stream, workspace))), "rlm_mix_backward")


def rlm_mix_backward_from(dy: torch.Tensor, x: torch.Tensor, params: Params, state_in: State | None,
                          d_state_out: State | None, dx: torch.Tensor, dparams: Grads,
                          d_state_in: State | None = None, workspace: torch.Tensor | None = None,
                          stream=None) -> None:
    """Backward of rlm_mix_prefill_from: dx, the parameter gradients and (if
    ``d_state_in`` is given) the gradient of the initial state, for a loss that may
    also depend on the terminal state (its gradient ``d_state_out``).  Only the
    ``s`` buffers of the state arguments are used."""
    lib = load_library()
    dyt, xt, dxt = _field(dy), _field(x), _field(dx)
    if workspace is None:
        workspace = _workspace(lib.rlm_backward_workspace_size(xt.B, xt.L, xt.D, params.M, xt.dtype),
                               x.device, stream)
    opt = lambda st: ctypes.byref(st._c()) if st is not None else None
    _check(lib.rlm_mix_backward_from(ctypes.byref(dyt), ctypes.byref(xt), ctypes.byref(params._c()),
                                     opt(state_in), opt(d_state_out), ctypes.byref(dxt),
                                     ctypes.byref(dparams._c()), opt(d_state_in),
                                     ctypes.byref(_launch(stream, workspace))), "rlm_mix_backward_from")


def rlm_validate_params(params: Params) -> None:
    _check(load_library().rlm_validate_params(ctypes.byref(params._c())), "rlm_validate_params")


def rlm_get_device_status(stream=None) -> int:
    """Synchronise the stream and return (and clear) the device status word."""
    return load_library().rlm_get_device_status(ctypes.byref(_launch(stream, None)))


def rlm_mixer_prefill(x: torch.Tensor, g: torch.Tensor | None, params: Params, local: Local | None,
                      z: torch.Tensor, state_in: State | None = None, conv_in: ConvState | None = None,
                      state_out: State | None = None, conv_out: ConvState | None = None,
                      workspace: torch.Tensor | None = None, stream=None,
                      coupling: Coupling | None = None) -> None:
    """Mixer output of Sec. 3.4 over a sequence: z = sigmoid(g) * y + s * (w * x), y the
    resonant mixing of x from ``state_in``; the local path reads its drives before
    token 0 from ``conv_in``.  ``state_out`` / ``conv_out`` receive the terminal
    state and drive history (each may be its input, for in-place continuation)."""
    lib = load_library()
    xt, zt = _field(x), _field(z)
    gt = _field(g) if g is not None else None
    if workspace is None:
        workspace = _workspace(lib.rlm_prefill_workspace_size(xt.B, xt.L, xt.D, params.M, xt.dtype),
                               x.device, stream)
    ref = lambda c: ctypes.byref(c) if c is not None else None
    opt = lambda o: ref(o._c()) if o is not None else None
    _check(lib.rlm_mixer_prefill(ctypes.byref(xt), ref(gt), ctypes.byref(params._c()), opt(local), opt(coupling),
                                 opt(state_in),
                                 opt(conv_in), ctypes.byref(zt), opt(state_out), opt(conv_out),
                                 ctypes.byref(_launch(stream, workspace))), "rlm_mixer_prefill")


def rlm_mixer_decode(x_t: torch.Tensor, g_t: torch.Tensor | None, state: State, local: Local | None,
                     conv: ConvState | None, z_t: torch.Tensor, stream=None, coupling: Coupling | None = None) -> None:
    """One mixer decode step: recurrence, gate and local path in one kernel; the state
    and the drive history advance in place."""
    lib = load_library()
    xt, zt = _field(x_t), _field(z_t)
    gt = _field(g_t) if g_t is not None else None
    ref = lambda c: ctypes.byref(c) if c is not None else None
    opt = lambda o: ref(o._c()) if o is not None else None
    _check(lib.rlm_mixer_decode(ctypes.byref(xt), ref(gt), ctypes.byref(state._c()), opt(local), opt(coupling),
                                opt(conv),
                                ctypes.byref(zt), ctypes.byref(_launch(stream, None))), "rlm_mixer_decode")


# ------------------------------------------------- gated linear recurrence
def rlm_scan_saved_size(B: int, L: int, D: int) -> int:
    return load_library().rlm_scan_saved_size(B, L, D)


SCAN_CHUNK = 64         # RLM_SCAN_CHUNK: tokens between the states a training pass keeps


def scan_saved(B: int, L: int, D: int, device="cuda") -> torch.Tensor:
    """A buffer for rlm_scan_prefill's ``saved``: float32 [B][ceil(L / 64)][D]."""
    return torch.empty(B, -(-L // SCAN_CHUNK), D, dtype=torch.float32, device=device)


def rlm_scan_prefill(x: torch.Tensor, g: torch.Tensor, y: torch.Tensor, leak: bool = True,
                     state_in: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                     saved: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                     stream=None) -> None:
    """Gated linear recurrence h_t = a_t h_{t-1} + i_t over a sequence, a = sigmoid(g),
    i = (1 - a) x (``leak``) or x; y receives every h_t.  Fields [B][L][D] may have row
    strides; states are float32 [B][D] (``state_out`` may be ``state_in``); ``lengths``
    int32 [B] marks padding; ``saved`` (see ``scan_saved``) keeps what the backward
    pass needs."""
    lib = load_library()
    xt, gt, yt = _strided(x, "x"), _strided(g, "g"), _strided(y, "y")
    B, L, D = xt.B, xt.L, xt.D
    _check(lib.rlm_scan_prefill(xt, gt, int(leak),
                                _opt(state_in, torch.float32, (B, D), "state_in"), yt,
                                _opt(state_out, torch.float32, (B, D), "state_out"),
                                _opt(saved, torch.float32, (B, -(-L // SCAN_CHUNK), D), "saved"),
                                _opt(lengths, torch.int32, (B,), "lengths"),
                                _launch(stream, None)), "rlm_scan_prefill")


def rlm_scan_backward(dy: torch.Tensor, x: torch.Tensor, g: torch.Tensor, saved: torch.Tensor, dx: torch.Tensor,
                      dg: torch.Tensor, leak: bool = True, d_state_out: torch.Tensor | None = None,
                      d_state_in: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                      stream=None) -> None:
    """Gradients of rlm_scan_prefill: dx, dg and (optionally) of its initial state, for a
    loss of y and, with ``d_state_out``, of the final state."""
    lib = load_library()
    dyt, xt, gt = _strided(dy, "dy"), _strided(x, "x"), _strided(g, "g")
    dxt, dgt = _strided(dx, "dx"), _strided(dg, "dg")
    B, L, D = xt.B, xt.L, xt.D
    _check(lib.rlm_scan_backward(dyt, xt, gt,
                                 _opt(saved, torch.float32, (B, -(-L // SCAN_CHUNK), D), "saved"), int(leak),
                                 _opt(d_state_out, torch.float32, (B, D), "d_state_out"), dxt,
                                 dgt, _opt(d_state_in, torch.float32, (B, D), "d_state_in"),
                                 _opt(lengths, torch.int32, (B,), "lengths"),
                                 _launch(stream, None)), "rlm_scan_backward")


def rlm_scan_decode(x_t: torch.Tensor, g_t: torch.Tensor, state: torch.Tensor, y_t: torch.Tensor, leak: bool = True,
                    stream=None) -> None:
    """One token of the gated linear recurrence; ``state`` (float32 [B][D]) advances in place."""
    xt, gt, yt = _strided(x_t, "x_t"), _strided(g_t, "g_t"), _strided(y_t, "y_t")
    _check(load_library().rlm_scan_decode(xt, gt, int(leak),
                                          _opt(state, torch.float32, (xt.B, xt.D), "state"), yt,
                                          _launch(stream, None)), "rlm_scan_decode")


# ------------------------------------------------------------ linear layer
ACTIVATIONS = {"none": 0, "silu": 1, "gelu": 2, "sigmoid": 3}


def _act(act: str) -> int:
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, got {act!r}")
    return ACTIVATIONS[act]


def rlm_linear_workspace_size(R: int, K: int, N: int) -> int:
    return load_library().rlm_linear_workspace_size(R, K, N)


def rlm_linear_backward_workspace_size(R: int, K: int, N: int, act: str = "none") -> int:
    return load_library().rlm_linear_backward_workspace_size(R, K, N, _act(act))


def rlm_linear(x: torch.Tensor, w: torch.Tensor, y: torch.Tensor, bias: torch.Tensor | None = None,
               residual: torch.Tensor | None = None, act: str = "none", pre: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None, stream=None) -> None:
    """y = act(x w^T + bias) + residual.  x [...][K], w [N][K], y and residual [...][N] bfloat16 (rows
    may be strided), bias float32 [N]; act is "none", "silu", "gelu" (tanh form) or "sigmoid".
    ``pre`` receives x w^T + bias for the backward pass; ``residual`` may be ``y`` itself."""
    lib = load_library()
    xt, wt, yt = _matrix(x, "x"), _matrix(w, "w"), _matrix(y, "y")
    rt = _matrix(residual, "residual") if residual is not None else None
    pt = _matrix(pre, "pre") if pre is not None else None
    if workspace is None:
        workspace = _workspace(lib.rlm_linear_workspace_size(xt.rows, xt.cols, wt.rows), x.device, stream)
    _check(lib.rlm_linear(xt, wt, _opt(bias, torch.float32, (wt.rows,), "bias"), _act(act),
                          rt, pt, yt, _launch(stream, workspace)), "rlm_linear")


def rlm_linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, dx: torch.Tensor | None = None,
                        dw: torch.Tensor | None = None, dbias: torch.Tensor | None = None, act: str = "none",
                        pre: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> None:
    """Gradients of rlm_linear: dx (bfloat16), dw (bfloat16 or float32) and dbias (float32), each
    optional.  ``pre`` is what the forward pass kept (needed unless act is "none")."""
    lib = load_library()
    dyt, xt, wt = _matrix(dy, "dy"), _matrix(x, "x"), _matrix(w, "w")
    opt = lambda t, name: _matrix(t, name) if t is not None else None
    pt, dxt, dwt = opt(pre, "pre"), opt(dx, "dx"), opt(dw, "dw")
    if workspace is None:
        workspace = _workspace(lib.rlm_linear_backward_workspace_size(xt.rows, xt.cols, wt.rows, _act(act)), x.device,
                               stream)
    _check(lib.rlm_linear_backward(dyt, xt, wt, pt, _act(act), dxt,
                                   dwt, _opt(dbias, torch.float32, (wt.rows,), "dbias"),
                                   _launch(stream, workspace)), "rlm_linear_backward")


# --------------------------------------------------------------- optimizer
ADAMW_BLOCK = 256       # RLM_ADAMW_BLOCK: values that share a scale of the 8-bit moments
ADAMW_DRAW = 0x100      # RLM_ADAMW_DRAW: 8-bit codes rounded by draw


@dataclass
class AdamState:
    """Moments of one tensor of n values: m and v float32 [n], or (8 bits) codes float8_e4m3fn
    [n] of m and of sqrt(v) with the scales float32 [ceil(n / 256)] of their blocks.

    ``draw`` says how a step rounds the codes: by draw, so that over many steps they follow the
    32-bit moments (what ``zeros`` sets, for training), or to nearest, where a change of less
    than half a code is lost (single steps from given moments)."""
    m: torch.Tensor
    v: torch.Tensor
    m_scale: torch.Tensor | None = None
    v_scale: torch.Tensor | None = None
    draw: bool = False

    @classmethod
    def zeros(cls, param: torch.Tensor, bits: int = 32):
        n, dev = param.numel(), param.device
        if bits == 32:
            return cls(*(torch.zeros(n, dtype=torch.float32, device=dev) for _ in range(2)))
        if bits != 8:
            raise ValueError(f"bits must be 8 or 32, got {bits}")
        k = -(-n // ADAMW_BLOCK)
        return cls(*(torch.zeros(n, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn) for _ in range(2)),
                   *(torch.ones(k, dtype=torch.float32, device=dev) for _ in range(2)), draw=True)

    @property
    def bits(self) -> int:
        return 32 if self.m.dtype == torch.float32 else 8

    def values(self) -> tuple[torch.Tensor, torch.Tensor]:
        """m and v as float32, whatever they are kept in."""
        if self.bits == 32:
            return self.m, self.v
        wide = lambda s: s.repeat_interleave(ADAMW_BLOCK)[: self.m.numel()]
        return self.m.float() * wide(self.m_scale), (self.v.float() * wide(self.v_scale)).square()


class AdamGroup:
    """The tensors of an optimizer step, checked and laid out once: weights (float32 or
    bfloat16), gradients (float32 or bfloat16), their AdamState and, for bfloat16 weights,
    optional float32 master copies.  It keeps the tensors; gradients are read from the same
    buffers at every step.  A gradient that is its weight's ``.grad`` has to stay it (zeroed in
    place, not set to None): a step raises ValueError where it no longer is."""

    def __init__(self, params, grads, states, masters=None):
        params, grads, states = list(params), list(grads), list(states)
        masters = [None] * len(params) if masters is None else list(masters)
        if not params or not len(params) == len(grads) == len(states) == len(masters):
            raise ValueError("AdamGroup needs as many grads, states (and masters) as params, and at least one")
        self.tensors = params, grads, states, masters
        self.param_dtype, self.grad_dtype, self.bits = params[0].dtype, grads[0].dtype, states[0].bits
        self.draw = bool(states[0].draw) and self.bits == 8
        if self.bits == 8 and any(bool(s.draw) != self.draw for s in states):
            raise ValueError("the states of a group are all rounded by draw or all to nearest")
        if self.param_dtype not in _DT or self.grad_dtype not in _DT:
            raise ValueError(f"weights are {self.param_dtype}, gradients {self.grad_dtype}: need float32 or bfloat16")
        self._c = (_AdamTensor * len(params))()
        self._watched = []              # weights whose .grad the group reads
        code = torch.float32 if self.bits == 32 else torch.float8_e4m3fn
        self.device = params[0].device
        for i, (p, g, s, w) in enumerate(zip(params, grads, states, masters)):
            n = p.numel()
            need = [(p, self.param_dtype, n, "weight"), (g, self.grad_dtype, n, "gradient"), (s.m, code, n, "m"),
                    (s.v, code, n, "v")]
            if w is not None:
                need.append((w, torch.float32, n, "master"))
            if self.bits == 8:
                k = -(-n // ADAMW_BLOCK)
                need += [(s.m_scale, torch.float32, k, "m_scale"), (s.v_scale, torch.float32, k, "v_scale")]
            for t, dtype, size, name in need:
                if t is None or t.dtype != dtype or t.numel() != size or not t.is_contiguous() or not t.is_cuda \
                        or t.device != self.device:
                    raise ValueError(f"tensor {i}: {name} must be a contiguous {dtype} tensor of {size} values on "
                                     f"{self.device}")
            if p.requires_grad and p.is_leaf and p.grad is not None and p.grad.data_ptr() == g.data_ptr():
                self._watched.append((i, p, g.data_ptr()))
            ptr = lambda t: t.data_ptr() if t is not None else None
            self._c[i] = _AdamTensor(ptr(p), ptr(g), ptr(s.m), ptr(s.v), ptr(s.m_scale) if self.bits == 8 else None,
                                     ptr(s.v_scale) if self.bits == 8 else None, ptr(w), n)


def rlm_adamw_step(group: AdamGroup, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999,
                   eps: float = 1e-8, weight_decay: float = 0.01, grad_scale: torch.Tensor | None = None,
                   stream=None) -> None:
    """One AdamW step (``step`` counts from 1) over a group's tensors, in place.  ``grad_scale``, a float32
    CUDA scalar, multiplies every gradient; a value that is not finite skips the step."""
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1 or not grad_scale.is_cuda):
        raise ValueError("grad_scale must be a CUDA float32 scalar")
    for i, p, grad in group._watched:
        if p.grad is None or p.grad.data_ptr() != grad:
            raise ValueError(f"tensor {i}: its weight's .grad is no longer the gradient that the group was given")
    h = _AdamHyper(lr, beta1, beta2, eps, weight_decay, step)
    _check(load_library().rlm_adamw_step(group._c, len(group._c), _DT[group.param_dtype], _DT[group.grad_dtype],
                                         group.bits | (ADAMW_DRAW if group.draw else 0), h,
                                         grad_scale.data_ptr() if grad_scale is not None else None,
                                         _launch(stream, None)), "rlm_adamw_step")
