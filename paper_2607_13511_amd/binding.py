"""Thin ctypes binding over ``libexternd.so`` (C ABI in ``include/externd.h``).

Argument marshalling only: torch tensors supply device memory and the
current HIP stream; every step of the factorization runs in the library's
HIP kernels.  There is no fallback: if the library is missing or no GPU is
present the calls raise.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libexternd.so")

OK, EINVAL, ENONFINITE, EWORKSPACE, EHIP, EUNSUPPORTED, ESYNC, ESCRATCH = 0, -1, -2, -3, -4, -5, -6, -7
APPLY_NOALLOC_MAX_BYTES = 8 << 20   # EXTERND_APPLY_NOALLOC_MAX_BYTES
MAX_BLOCK = 256

_lib = None

_c_i64 = ctypes.c_int64
_c_i32 = ctypes.c_int32
_c_dbl = ctypes.c_double
_c_ptr = ctypes.c_void_p
_c_size = ctypes.c_size_t

# name -> (restype, argtypes)
_SIGNATURES = {
    "externd_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "externd_rank": (_c_i64, [_c_i64, _c_i64, _c_dbl]),
    "externd_effective_block": (_c_i32, [_c_i64, _c_i64, _c_i32]),
    "externd_workspace_bytes": (_c_size, [_c_i64, _c_i64, _c_i64]),
    "externd_factorize": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_dbl, _c_dbl, _c_i32, _c_i32, _c_ptr,
                                         _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr,
                                         _c_ptr, _c_size, _c_ptr]),
    "externd_factorize_ex": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_dbl, _c_dbl, _c_i32, _c_i32, _c_ptr,
                                            _c_dbl, _c_i32, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr,
                                            _c_ptr, _c_ptr, _c_size, _c_ptr]),
    "externd_factorize_to_energy": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_dbl, _c_dbl, _c_dbl, _c_i32, _c_i32,
                                                   _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr,
                                                   _c_ptr, _c_ptr, _c_size, _c_ptr]),
    "externd_factorize_refined": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_dbl, _c_dbl, _c_i32, _c_i32, _c_i32,
                                                 _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr,
                                                 _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_size, _c_ptr]),
    "externd_apply_workspace_bytes": (_c_size, [_c_i64, _c_i64, _c_i64, _c_i32]),
    "externd_apply": (ctypes.c_int, [_c_ptr, _c_ptr, _c_ptr, _c_i64, _c_i64, _c_i64, _c_ptr, _c_i32, _c_ptr,
                                     _c_ptr, _c_size, _c_ptr]),
    "externd_apply_noalloc": (ctypes.c_int, [_c_ptr, _c_ptr, _c_ptr, _c_i64, _c_i64, _c_i64, _c_ptr, _c_i32,
                                             _c_ptr, _c_ptr]),
    "externd_factorize_timed": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_dbl, _c_dbl, _c_i32, _c_i32, _c_ptr,
                                               _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr,
                                               _c_ptr, _c_size, _c_ptr, _c_ptr]),
    "externd_step_init": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_ptr, _c_i32, _c_dbl, _c_ptr, _c_ptr,
                                         _c_ptr, _c_size, _c_ptr]),
    "externd_step_vstep": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_ptr, _c_i32, _c_dbl, _c_ptr, _c_ptr,
                                          _c_ptr, _c_size, _c_ptr]),
    "externd_step_ustep": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_ptr, _c_i32, _c_dbl, _c_ptr, _c_ptr,
                                          _c_ptr, _c_ptr, _c_ptr, _c_size, _c_ptr]),
    "externd_step_scale": (ctypes.c_int, [_c_ptr, _c_ptr, _c_ptr, _c_i64, _c_i64, _c_i32, _c_ptr, _c_ptr,
                                          _c_ptr, _c_size, _c_ptr]),
    "externd_step_deflate": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_ptr, _c_ptr, _c_ptr, _c_i32,
                                            _c_ptr, _c_ptr, _c_ptr, _c_size, _c_ptr]),
    "externd_rotary_frequencies": (ctypes.c_int, [_c_i32, _c_dbl, _c_i32, _c_dbl, _c_i64, _c_dbl, _c_dbl, _c_ptr,
                                                  _c_ptr]),
    "externd_rotary": (ctypes.c_int, [_c_ptr, _c_ptr, _c_i64, _c_i64, _c_i64, _c_i64, _c_i32, _c_ptr, _c_ptr, _c_i64,
                                      _c_i64, _c_i64, _c_i64, _c_i32, _c_i32, _c_i64, _c_i32, _c_i32, _c_i32, _c_i32,
                                      _c_ptr, _c_ptr, ctypes.c_float, _c_ptr]),
    "externd_kv4_page_bytes": (_c_size, [_c_i32, _c_i32]),
    "externd_kv4_append": (ctypes.c_int, [_c_ptr, _c_i64, _c_i32, _c_i32, _c_i32, _c_ptr, _c_ptr, _c_i32, _c_i64,
                                          _c_i64, _c_i64, _c_i64, _c_i64, _c_i32, _c_ptr, _c_ptr, _c_ptr, _c_i64,
                                          _c_ptr]),
    "externd_kv4_read": (ctypes.c_int, [_c_ptr, _c_i64, _c_i32, _c_i32, _c_i32, _c_ptr, _c_ptr, _c_i32, _c_i64,
                                        _c_i32, _c_ptr, _c_ptr, _c_ptr, _c_i64, _c_ptr]),
    "externd_kv4_attention_workspace_bytes": (_c_size, [_c_i32, _c_i32, _c_i32, _c_i32, _c_i64, _c_i32, _c_i32,
                                                        _c_i64]),
    "externd_kv4_attention_block_rows": (_c_i32, [_c_i32, _c_i32, _c_i32, _c_i32, _c_i64, _c_i32, _c_i32, _c_i64]),
    "externd_kv4_attention": (ctypes.c_int, [_c_ptr, _c_i64, _c_i32, _c_i32, _c_i32, _c_ptr, _c_i32, _c_i64, _c_i64,
                                             _c_i32, _c_ptr, _c_ptr, _c_i64, _c_i32, _c_i32, _c_i64, _c_ptr, _c_ptr,
                                             _c_ptr, _c_i64, ctypes.c_float, _c_i32, _c_ptr, _c_size, _c_ptr]),
    "externd_token_logprobs_workspace_bytes": (_c_size, [_c_i64, _c_i64, _c_i32]),
    "externd_token_logprobs": (ctypes.c_int, [_c_ptr, _c_i32, _c_i64, _c_i64, _c_i64, _c_ptr, ctypes.c_float, _c_i32,
                                              _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_size, _c_ptr]),
    "externd_token_logprobs_backward": (ctypes.c_int, [_c_ptr, _c_i32, _c_i64, _c_i64, _c_i64, _c_ptr, ctypes.c_float,
                                                       _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_i64, _c_ptr]),
    "externd_embedding": (ctypes.c_int, [_c_ptr, _c_i32, _c_i64, _c_i64, _c_i64, _c_ptr, _c_i64, ctypes.c_float, _c_ptr,
                                         _c_i64, _c_ptr]),
    "externd_embedding_backward_workspace_bytes": (_c_size, [_c_i64, _c_i64, _c_i64]),
    "externd_embedding_backward": (ctypes.c_int, [_c_ptr, _c_i32, _c_i64, _c_i64, _c_i64, _c_ptr, _c_i64, ctypes.c_float,
                                                  _c_i32, _c_ptr, _c_i64, _c_ptr, _c_size, _c_ptr]),
    "externd_linear_logprobs_workspace_bytes": (_c_size, [_c_i32, _c_i64, _c_i64, _c_i64]),
    "externd_linear_logprobs": (ctypes.c_int, [_c_ptr, _c_i64, _c_ptr, _c_i64, _c_i32, _c_i64, _c_i64, _c_i64, _c_ptr,
                                               ctypes.c_float, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_size, _c_ptr]),
    "externd_linear_logprobs_backward_workspace_bytes": (_c_size, [_c_i32, _c_i64, _c_i64, _c_i64, _c_i32, _c_i32]),
    "externd_linear_logprobs_backward": (ctypes.c_int, [_c_ptr, _c_i64, _c_ptr, _c_i64, _c_i32, _c_i64, _c_i64, _c_i64,
                                                        _c_ptr, ctypes.c_float, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_ptr,
                                                        _c_i64, _c_ptr, _c_i64, _c_ptr, _c_size, _c_ptr]),
    "externd_clip_gradients_workspace_bytes": (_c_size, [_c_i64]),
    "externd_clip_gradients": (ctypes.c_int, [_c_i64, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_dbl, _c_ptr, _c_ptr, _c_size,
                                              _c_ptr]),
}
EXPORTED = tuple(_SIGNATURES)


KCLASS_NAMES = ("vstep_contraction", "ustep_contraction", "deflate", "vstep_target", "ustep_target",
                "sequential_one_launch", "ternarize_v", "ternarize_u")
# externd_factorize_timed times one launch in TIMING_STRIDE of each class
# (EXTERND_TIMING_STRIDE in include/externd.h).
TIMING_STRIDE = 16


class KernelTimes(ctypes.Structure):
    _fields_ = [("total_ms", ctypes.c_double * len(KCLASS_NAMES)), ("launches", ctypes.c_int64 * len(KCLASS_NAMES)),
                ("issued", ctypes.c_int64 * len(KCLASS_NAMES))]


class ExterndError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().externd_strerror(status).decode()
        super().__init__(f"{where}: {msg} (status {status})")


def lib():
    """Load the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != OK:
        raise ExterndError(status, where)


def rank(m: int, n: int, mu: float) -> int:
    return int(lib().externd_rank(m, n, mu))


def effective_block(m: int, n: int, block: int) -> int:
    return int(lib().externd_effective_block(m, n, block))


def workspace_bytes(m: int, n: int, k: int = 0) -> int:
    return int(lib().externd_workspace_bytes(m, n, k))


# ---------------------------------------------------------------------------
# torch marshalling
# ---------------------------------------------------------------------------
_torch_module = None   # torch, once a GPU has been seen


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("externd needs a HIP GPU (torch.cuda is not available)")
        _torch_module = torch
    return _torch_module


def _dev_ptr(t) -> int:
    return int(t.data_ptr())


def _stream_ptr(torch, stream) -> int:
    if stream is None:
        # the current stream's handle without building a Stream object for it
        # (1 us of a small call), where this torch has those private functions
        raw, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and dev is not None:
            return raw(dev())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _workspace(torch, m, n, k, device):
    nbytes = workspace_bytes(m, n, k)
    if nbytes == 0:
        raise ExterndError(EUNSUPPORTED, "workspace_bytes")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _req(t, torch, dtype, shape, name):
    if not (t.is_cuda and t.dtype is dtype and t.is_contiguous() and t.shape == shape):
        raise ValueError(f"{name}: expected a contiguous {dtype} CUDA tensor of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


@dataclass
class Factorization:
    B_packed: "object"        # torch.uint8 (m, ceil(k/4))
    C_packed: "object"        # torch.uint8 (k, ceil(n/4))
    D: "object"               # torch.float32 (k,)
    E: float
    E_w: float
    curve: np.ndarray
    curve_w: np.ndarray
    k: int
    block: int
    kernel_times: Optional[dict] = None   # class -> (total_ms, timed launches, all launches) when timed
    k_used: int = -1                      # components extracted (factorize_to_energy), else k
    safeguard_fired: int = 0              # blocks replaced by the single-entry step (factorize_ex)


def factorize(A, mu: float, tau: float, block: int, iters: int, h=None, stream=None,
              workspace=None, timed: bool = False) -> Factorization:
    """Factorize the fp32 CUDA tensor A (m x n) as B diag(D) C on the GPU.

    With ``timed`` the library records HIP events around every contraction
    and deflation launch and returns their summed durations.
    """
    torch = _torch()
    m, n = A.shape
    _req(A, torch, torch.float32, (m, n), "A")
    if h is not None:
        _req(h, torch, torch.float32, (n,), "h")
    k = rank(m, n, mu)
    if k < 1:
        raise ExterndError(EINVAL, "rank")
    b = effective_block(m, n, block)
    nblk = -(-k // b)
    dev = A.device
    Bp = torch.empty((m, (k + 3) // 4), dtype=torch.uint8, device=dev)
    Cp = torch.empty((k, (n + 3) // 4), dtype=torch.uint8, device=dev)
    D = torch.empty((k,), dtype=torch.float32, device=dev)
    ws = workspace if workspace is not None else _workspace(torch, m, n, k, dev)
    E = ctypes.c_double(0.0)
    Ew = ctypes.c_double(0.0)
    curve = np.zeros(nblk, dtype=np.float64)
    curve_w = np.zeros(nblk, dtype=np.float64)
    args = (_dev_ptr(A), m, n, mu, tau, block, iters, _dev_ptr(h) if h is not None else None,
            _dev_ptr(Bp), _dev_ptr(Cp), _dev_ptr(D), ctypes.byref(E), ctypes.byref(Ew),
            curve.ctypes.data, curve_w.ctypes.data, _dev_ptr(ws), ws.numel(), _stream_ptr(torch, stream))
    kt = None
    if timed:
        times = KernelTimes()
        _check(lib().externd_factorize_timed(*args, ctypes.byref(times)), "externd_factorize_timed")
        kt = {name: (times.total_ms[i], int(times.launches[i]), int(times.issued[i]))
              for i, name in enumerate(KCLASS_NAMES)}
    else:
        _check(lib().externd_factorize(*args), "externd_factorize")
    return Factorization(Bp, Cp, D, E.value, Ew.value, curve, curve_w, k, b, kt, k)


def factorize_ex(A, mu: float, tau: float, block: int, iters: int, h=None, lam: float = 0.0,
                 safeguard: bool = False, stream=None, workspace=None) -> Factorization:
    """externd_factorize with the lambda of the importance weights
    (h~ = h / max h + lam) and the single-entry safeguard of Proposition 2
    (plain objective only) (externd_factorize_ex)."""
    torch = _torch()
    m, n = A.shape
    _req(A, torch, torch.float32, (m, n), "A")
    if h is not None:
        _req(h, torch, torch.float32, (n,), "h")
    k = rank(m, n, mu)
    if k < 1:
        raise ExterndError(EINVAL, "rank")
    b = effective_block(m, n, block)
    nblk = -(-k // b)
    dev = A.device
    Bp = torch.empty((m, (k + 3) // 4), dtype=torch.uint8, device=dev)
    Cp = torch.empty((k, (n + 3) // 4), dtype=torch.uint8, device=dev)
    D = torch.empty((k,), dtype=torch.float32, device=dev)
    ws = workspace if workspace is not None else _workspace(torch, m, n, k, dev)
    E = ctypes.c_double(0.0)
    Ew = ctypes.c_double(0.0)
    fired = ctypes.c_int64(0)
    curve = np.zeros(nblk, dtype=np.float64)
    curve_w = np.zeros(nblk, dtype=np.float64)
    _check(lib().externd_factorize_ex(
        _dev_ptr(A), m, n, mu, tau, block, iters, _dev_ptr(h) if h is not None else None, lam, int(safeguard),
        _dev_ptr(Bp), _dev_ptr(Cp), _dev_ptr(D), ctypes.byref(E), ctypes.byref(Ew), curve.ctypes.data,
        curve_w.ctypes.data, ctypes.byref(fired), _dev_ptr(ws), ws.numel(), _stream_ptr(torch, stream)),
        "externd_factorize_ex")
    return Factorization(Bp, Cp, D, E.value, Ew.value, curve, curve_w, k, b, None, k, int(fired.value))


APPLY_MAX_BATCH = 8   # EXTERND_APPLY_MAX_BATCH


def apply(B_packed, C_packed, D, m: int, n: int, X, stream=None, workspace=None):
    """Y = X (B diag(D) C)^T on the GPU for the nb <= 8 rows of the fp32 CUDA
    tensor X (nb x n), from packed factors (externd_apply).  Returns Y (nb x m)."""
    torch = _torch()
    k = D.shape[0]
    nb = X.shape[0]
    _req(X, torch, torch.float32, (nb, n), "X")
    _req(D, torch, torch.float32, (k,), "D")
    _req(B_packed, torch, torch.uint8, (m, (k + 3) // 4), "B_packed")
    _req(C_packed, torch, torch.uint8, (k, (n + 3) // 4), "C_packed")
    Y = torch.empty((nb, m), dtype=torch.float32, device=X.device)
    L = lib()
    # the library checks a given workspace's size itself
    if workspace is None or not 1 <= nb <= APPLY_MAX_BATCH or max(m, n, k) > 1 << 31:
        nbytes = L.externd_apply_workspace_bytes(m, n, k, nb)
        if nbytes == 0:
            raise ExterndError(EINVAL, "externd_apply_workspace_bytes")
    ws = workspace if workspace is not None else torch.empty(nbytes, dtype=torch.uint8, device=X.device)
    st = L.externd_apply(B_packed.data_ptr(), C_packed.data_ptr(), D.data_ptr(), m, n, k, X.data_ptr(), nb,
                         Y.data_ptr(), ws.data_ptr(), ws.numel(), _stream_ptr(torch, stream))
    if st != OK:
        raise ExterndError(st, "externd_apply")
    return Y


def apply_noalloc(B_packed, C_packed, D, m: int, n: int, X, Y=None, stream=None):
    """As ``apply`` through externd_apply_noalloc: no workspace, the
    workspace lives in the library's fixed per-device scratch.  ``Y``
    (nb x m fp32 CUDA tensor) may be given so that the call allocates
    nothing at all.  Returns Y."""
    torch = _torch()
    k = D.shape[0]
    nb = X.shape[0]
    _req(X, torch, torch.float32, (nb, n), "X")
    _req(D, torch, torch.float32, (k,), "D")
    _req(B_packed, torch, torch.uint8, (m, (k + 3) // 4), "B_packed")
    _req(C_packed, torch, torch.uint8, (k, (n + 3) // 4), "C_packed")
    if Y is None:
        Y = torch.empty((nb, m), dtype=torch.float32, device=X.device)
    _req(Y, torch, torch.float32, (nb, m), "Y")
    _check(lib().externd_apply_noalloc(_dev_ptr(B_packed), _dev_ptr(C_packed), _dev_ptr(D), m, n, k, _dev_ptr(X),
                                       nb, _dev_ptr(Y), _stream_ptr(torch, stream)), "externd_apply_noalloc")
    return Y


def factorize_to_energy(A, mu_max: float, target: float, tau: float, block: int, iters: int, h=None,
                        stream=None, workspace=None) -> Factorization:
    """Factorize A until the energy (E, or E_w with h) reaches ``target``,
    with at most rank(m, n, mu_max) components (externd_factorize_to_energy).
    The result is sized for the maximum; components past ``k_used`` are
    zero and ``curve`` holds the blocks extracted."""
    torch = _torch()
    m, n = A.shape
    _req(A, torch, torch.float32, (m, n), "A")
    if h is not None:
        _req(h, torch, torch.float32, (n,), "h")
    k = rank(m, n, mu_max)
    if k < 1:
        raise ExterndError(EINVAL, "rank")
    b = effective_block(m, n, block)
    nblk = -(-k // b)
    dev = A.device
    Bp = torch.empty((m, (k + 3) // 4), dtype=torch.uint8, device=dev)
    Cp = torch.empty((k, (n + 3) // 4), dtype=torch.uint8, device=dev)
    D = torch.empty((k,), dtype=torch.float32, device=dev)
    ws = workspace if workspace is not None else _workspace(torch, m, n, k, dev)
    E = ctypes.c_double(0.0)
    Ew = ctypes.c_double(0.0)
    ku = ctypes.c_int64(0)
    curve = np.zeros(nblk, dtype=np.float64)
    curve_w = np.zeros(nblk, dtype=np.float64)
    _check(lib().externd_factorize_to_energy(
        _dev_ptr(A), m, n, mu_max, target, tau, block, iters, _dev_ptr(h) if h is not None else None,
        _dev_ptr(Bp), _dev_ptr(Cp), _dev_ptr(D), ctypes.byref(ku), ctypes.byref(E), ctypes.byref(Ew),
        curve.ctypes.data, curve_w.ctypes.data, _dev_ptr(ws), ws.numel(), _stream_ptr(torch, stream)),
        "externd_factorize_to_energy")
    nb = -(-ku.value // b)
    return Factorization(Bp, Cp, D, E.value, Ew.value, curve[:nb], curve_w[:nb], k, b, None, int(ku.value))


@dataclass
class Refined:
    factorization: Factorization       # final factors; E, E_w after the last sweep; extraction curve
    sweep_curve: np.ndarray            # E after each sweep
    sweep_curve_w: np.ndarray          # weighted E after each sweep
    accepted: int                      # revisits that replaced their block
    revisits: int


def factorize_refined(A, mu: float, tau: float, block: int, iters: int, sweeps: int, h=None, stream=None,
                      workspace=None) -> Refined:
    """Factorize A, then run ``sweeps`` refinement sweeps over its blocks
    (externd_factorize_refined)."""
    torch = _torch()
    m, n = A.shape
    _req(A, torch, torch.float32, (m, n), "A")
    if h is not None:
        _req(h, torch, torch.float32, (n,), "h")
    k = rank(m, n, mu)
    if k < 1:
        raise ExterndError(EINVAL, "rank")
    b = effective_block(m, n, block)
    nblk = -(-k // b)
    dev = A.device
    Bp = torch.empty((m, (k + 3) // 4), dtype=torch.uint8, device=dev)
    Cp = torch.empty((k, (n + 3) // 4), dtype=torch.uint8, device=dev)
    D = torch.empty((k,), dtype=torch.float32, device=dev)
    ws = workspace if workspace is not None else _workspace(torch, m, n, k, dev)
    E = ctypes.c_double(0.0)
    Ew = ctypes.c_double(0.0)
    acc = ctypes.c_int64(0)
    curve = np.zeros(nblk, dtype=np.float64)
    curve_w = np.zeros(nblk, dtype=np.float64)
    sc = np.zeros(max(sweeps, 1), dtype=np.float64)
    scw = np.zeros(max(sweeps, 1), dtype=np.float64)
    _check(lib().externd_factorize_refined(
        _dev_ptr(A), m, n, mu, tau, block, iters, sweeps, _dev_ptr(h) if h is not None else None,
        _dev_ptr(Bp), _dev_ptr(Cp), _dev_ptr(D), ctypes.byref(E), ctypes.byref(Ew),
        curve.ctypes.data, curve_w.ctypes.data, sc.ctypes.data, scw.ctypes.data, ctypes.byref(acc),
        _dev_ptr(ws), ws.numel(), _stream_ptr(torch, stream)), "externd_factorize_refined")
    F = Factorization(Bp, Cp, D, E.value, Ew.value, curve, curve_w, k, b, None, k)
    return Refined(F, sc[:sweeps], scw[:sweeps], int(acc.value), sweeps * nblk)


def step_init(R, bb: int, tau: float, h=None, stream=None):
    torch = _torch()
    m, n = R.shape
    _req(R, torch, torch.float32, (m, n), "R")
    U = torch.empty((m, bb), dtype=torch.int8, device=R.device)
    J = torch.empty((bb,), dtype=torch.int32, device=R.device)
    ws = _workspace(torch, m, n, 0, R.device)
    st = lib().externd_step_init(_dev_ptr(R), m, n, _dev_ptr(h) if h is not None else None, bb, tau,
                                 _dev_ptr(U), _dev_ptr(J), _dev_ptr(ws), ws.numel(), _stream_ptr(torch, stream))
    _check(st, "externd_step_init")
    return U, J


def step_vstep(R, U, tau: float, stream=None):
    torch = _torch()
    m, n = R.shape
    bb = U.shape[1]
    _req(R, torch, torch.float32, (m, n), "R")
    _req(U, torch, torch.int8, (m, bb), "U")
    V = torch.empty((n, bb), dtype=torch.int8, device=R.device)
    Y = torch.empty((bb, n), dtype=torch.float64, device=R.device)
    ws = _workspace(torch, m, n, 0, R.device)
    st = lib().externd_step_vstep(_dev_ptr(R), m, n, _dev_ptr(U), bb, tau, _dev_ptr(V), _dev_ptr(Y),
                                  _dev_ptr(ws), ws.numel(), _stream_ptr(torch, stream))
    _check(st, "externd_step_vstep")
    return V, Y


def step_ustep(R, V, tau: float, h=None, stream=None):
    torch = _torch()
    m, n = R.shape
    bb = V.shape[1]
    _req(R, torch, torch.float32, (m, n), "R")
    _req(V, torch, torch.int8, (n, bb), "V")
    U = torch.empty((m, bb), dtype=torch.int8, device=R.device)
    Q = torch.empty((m, bb), dtype=torch.float64, device=R.device)
    Z = torch.empty((m, bb), dtype=torch.float64, device=R.device)
    ws = _workspace(torch, m, n, 0, R.device)
    st = lib().externd_step_ustep(_dev_ptr(R), m, n, _dev_ptr(V), bb, tau, _dev_ptr(h) if h is not None else None,
                                  _dev_ptr(U), _dev_ptr(Q), _dev_ptr(Z), _dev_ptr(ws), ws.numel(),
                                  _stream_ptr(torch, stream))
    _check(st, "externd_step_ustep")
    return U, Q, Z


def step_scale(U, V, Q, h=None, stream=None):
    torch = _torch()
    m, bb = U.shape
    n = V.shape[0]
    _req(U, torch, torch.int8, (m, bb), "U")
    _req(V, torch, torch.int8, (n, bb), "V")
    _req(Q, torch, torch.float64, (m, bb), "Q")
    d = torch.empty((bb,), dtype=torch.float64, device=U.device)
    ws = _workspace(torch, m, n, 0, U.device)
    st = lib().externd_step_scale(_dev_ptr(U), _dev_ptr(V), _dev_ptr(Q), m, n, bb,
                                  _dev_ptr(h) if h is not None else None, _dev_ptr(d), _dev_ptr(ws), ws.numel(),
                                  _stream_ptr(torch, stream))
    _check(st, "externd_step_scale")
    return d


def step_deflate(R, U, V, d, stream=None):
    """In-place R <- R - U diag(fp32(d)) V^T; returns (colnorm2, fro2)."""
    torch = _torch()
    m, n = R.shape
    bb = U.shape[1]
    _req(R, torch, torch.float32, (m, n), "R")
    _req(U, torch, torch.int8, (m, bb), "U")
    _req(V, torch, torch.int8, (n, bb), "V")
    _req(d, torch, torch.float64, (bb,), "d")
    col = torch.empty((n,), dtype=torch.float64, device=R.device)
    fro = torch.empty((1,), dtype=torch.float64, device=R.device)
    ws = _workspace(torch, m, n, 0, R.device)
    st = lib().externd_step_deflate(_dev_ptr(R), m, n, _dev_ptr(U), _dev_ptr(V), _dev_ptr(d), bb, _dev_ptr(col),
                                    _dev_ptr(fro), _dev_ptr(ws), ws.numel(), _stream_ptr(torch, stream))
    _check(st, "externd_step_deflate")
    return col, fro


# ---------------------------------------------------------------------------
# operators of decoding: rotary positions, the 4-bit cache and attention over
# it, log probabilities of given tokens
# ---------------------------------------------------------------------------
ROPE_SCALINGS = ("plain", "linear", "base", "parts")   # EXTERND_ROPE_*
LOGPROBS_MAX_TOP = 64                                  # EXTERND_LOGPROBS_MAX_TOP
_dtype_codes = None   # torch dtype -> EXTERND_F32, _BF16, _F16


def _dtype_code(torch, dtype, name) -> int:
    global _dtype_codes
    if _dtype_codes is None:
        _dtype_codes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    code = _dtype_codes.get(dtype)
    if code is None:
        raise ValueError(f"{name}: expected float32, bfloat16 or float16, got {dtype}")
    return code


def _req_heads(t, dtype, tokens, name):
    """A CUDA tensor (tokens, heads, channels) of dtype whose channels are dense; returns its token and head strides."""
    if not (t.is_cuda and t.dtype is dtype and t.dim() == 3 and t.shape[0] == tokens):
        raise ValueError(f"{name}: expected a {dtype} CUDA tensor of shape ({tokens}, heads, channels), "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    ts, hs, cs = t.stride()
    if cs != 1 and t.shape[2] > 1:
        raise ValueError(f"{name}: the channels of a head must be dense, got strides {t.stride()}")
    return ts, hs


def rotary_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                       original_length: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """Frequencies of the rot_dim / 2 pairs as an int64 numpy array in units
    of 2^-64 turns a position, and the amplitude of the turned entries
    (externd_rotary_frequencies).  Needs no GPU."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling: expected one of {ROPE_SCALINGS}, got {scaling!r}")
    freqs = np.zeros(max(rot_dim // 2, 1), dtype=np.int64)
    amplitude = ctypes.c_double(0.0)
    _check(lib().externd_rotary_frequencies(rot_dim, base, ROPE_SCALINGS.index(scaling), factor, original_length,
                                            beta_fast, beta_slow, freqs.ctypes.data, ctypes.byref(amplitude)),
           "externd_rotary_frequencies")
    return freqs, amplitude.value


def _rotary(q, k, positions, freqs, interleaved, amplitude, inverse, out, stream):
    torch = _torch()
    if stream is not None:      # as on that stream: its own memory for what is allocated here
        with torch.cuda.stream(stream):
            return _rotary(q, k, positions, freqs, interleaved, amplitude, inverse, out, None)
    if q.dim() != 3:
        raise ValueError(f"q: expected (tokens, heads, channels), got shape {tuple(q.shape)}")
    tokens, heads, dim = q.shape
    code = _dtype_code(torch, q.dtype, "q")
    qs = _req_heads(q, q.dtype, tokens, "q")
    _req(positions, torch, torch.int64, (tokens,), "positions")
    half = freqs.numel()
    _req(freqs, torch, torch.int64, (half,), "freqs")
    ks = kos = (0, 0)
    ko = kp = kop = None
    kh = 0
    if k is not None:
        ks = _req_heads(k, q.dtype, tokens, "k")
        kh = k.shape[1]
        if k.shape[2] != dim:
            raise ValueError(f"k: expected {dim} channels a head, got {k.shape[2]}")
        kp = k.data_ptr()
    if out is None:
        qo, qos = q.new_empty((tokens, heads, dim)), (heads * dim, dim)
        if kh:
            ko, kos = q.new_empty((tokens, kh, dim)), (kh * dim, dim)
    else:
        qo, ko = out
        qos = _req_heads(qo, q.dtype, tokens, "q out")
        if qo.shape != q.shape:
            raise ValueError(f"q out: expected shape {tuple(q.shape)}, got {tuple(qo.shape)}")
        if kh:
            if ko is None or ko.shape != k.shape:
                raise ValueError(f"k out: expected shape {tuple(k.shape)}")
            kos = _req_heads(ko, q.dtype, tokens, "k out")
    if kh:
        kop = ko.data_ptr()
    if tokens:
        st = lib().externd_rotary(q.data_ptr(), qo.data_ptr(), qs[0], qs[1], qos[0], qos[1], heads, kp, kop, ks[0],
                                  ks[1], kos[0], kos[1], kh, code, tokens, dim, 2 * half, int(interleaved),
                                  inverse, positions.data_ptr(), freqs.data_ptr(), amplitude,
                                  _stream_ptr(torch, stream))
        if st != OK:
            raise ExterndError(st, "externd_rotary")
    return qo, ko


def rotary(q, k, positions, freqs, interleaved: bool = False, amplitude: float = 1.0, out=None, stream=None):
    """q and k (tokens x heads x channels; k may be None) turned to their
    int64 positions (externd_rotary).  ``freqs``: CUDA int64, as
    ``rotary_frequencies`` gives them; the first 2 * len(freqs) channels of a
    head are turned.  ``out``: (q_out, k_out), which may be (q, k) themselves.
    Returns (q', k')."""
    return _rotary(q, k, positions, freqs, interleaved, amplitude, 0, out, stream)


def rotary_backward(grad_q, grad_k, positions, freqs, interleaved: bool = False, amplitude: float = 1.0, out=None,
                    stream=None):
    """Gradients for q and k from those of ``rotary``'s results: the inverse
    turn with the same amplitude (externd_rotary)."""
    return _rotary(grad_q, grad_k, positions, freqs, interleaved, amplitude, 1, out, stream)


def kv4_cache(num_pages: int, heads_kv: int, head_dim: int, page_tokens: int, device="cuda"):
    """An empty cache in 4 bits: uint8 (num_pages, heads_kv, bytes of a page
    and head)."""
    torch = _torch()
    nbytes = lib().externd_kv4_page_bytes(head_dim, page_tokens)
    if nbytes == 0:
        raise ExterndError(EINVAL, "externd_kv4_page_bytes")
    return torch.zeros((num_pages, heads_kv, nbytes), dtype=torch.uint8, device=device)


def _kv4_args(torch, cache, head_dim, tokens, table, lens, starts):
    """(num_pages, heads, page tokens, batch, starts pointer) of a call on a cache."""
    if not (cache.is_cuda and cache.dtype is torch.uint8 and cache.dim() == 3 and cache.is_contiguous()):
        raise ValueError(f"cache: expected a contiguous uint8 CUDA tensor (pages, heads, bytes), got {cache.dtype} "
                         f"{tuple(cache.shape)} on {cache.device}")
    pages, heads, nbytes = cache.shape
    per = head_dim + head_dim // 16
    if head_dim not in (64, 128, 256) or nbytes % per:
        raise ValueError(f"cache: {nbytes} bytes a page and head are no whole number of tokens of {head_dim} channels")
    batch = lens.numel()
    _req(lens, torch, torch.int32, (batch,), "lens")
    if not (table.is_cuda and table.dtype is torch.int32 and table.dim() == 2 and table.shape[0] == batch
            and table.is_contiguous()):
        raise ValueError(f"table: expected a contiguous int32 CUDA tensor ({batch}, pages), got {table.dtype} "
                         f"{tuple(table.shape)} on {table.device}")
    sp = None
    if starts is not None:
        _req(starts, torch, torch.int32, (batch + 1,), "starts")
        sp = starts.data_ptr()
    elif tokens != batch:
        raise ValueError(f"without starts there is one new token a sequence: {tokens} tokens, {batch} sequences")
    return pages, heads, nbytes // per, batch, sp


def kv4_append(cache, k, v, table, lens, starts=None, stream=None):
    """Stores k and v (new tokens x cache heads x channels) in the cache, in
    place (externd_kv4_append).  ``lens`` int32: tokens of each sequence with
    the new ones; ``table`` int32 (sequences, pages): their pages; ``starts``
    int32 (sequences + 1): where each sequence's new tokens are, or None for
    one each."""
    torch = _torch()
    if k.dim() != 3 or v.shape != k.shape:
        raise ValueError(f"k, v: expected the same (tokens, heads, channels), got {tuple(k.shape)} and {tuple(v.shape)}")
    tokens, heads, dim = k.shape
    pages, kv, page, batch, sp = _kv4_args(torch, cache, dim, tokens, table, lens, starts)
    if heads != kv:
        raise ValueError(f"k, v: expected the cache's {kv} heads, got {heads}")
    code = _dtype_code(torch, k.dtype, "k")
    ks, vs = _req_heads(k, k.dtype, tokens, "k"), _req_heads(v, k.dtype, tokens, "v")
    if tokens:
        st = lib().externd_kv4_append(cache.data_ptr(), pages, kv, dim, page, k.data_ptr(), v.data_ptr(), code, ks[0],
                                      ks[1], vs[0], vs[1], tokens, batch, sp, lens.data_ptr(), table.data_ptr(),
                                      table.shape[1], _stream_ptr(torch, stream))
        if st != OK:
            raise ExterndError(st, "externd_kv4_append")


def kv4_read(cache, table, lens, head_dim: int, starts=None, tokens=None, dtype=None, stream=None):
    """K and V (tokens x cache heads x channels) as the cache holds them for
    the new tokens that ``starts`` (and their number ``tokens``) names; with
    starts over whole sequences, for all tokens (externd_kv4_read)."""
    torch = _torch()
    if stream is not None:      # as on that stream: its own memory for what is allocated here
        with torch.cuda.stream(stream):
            return kv4_read(cache, table, lens, head_dim, starts, tokens, dtype)
    if tokens is None:
        if starts is not None:
            raise ValueError("tokens: their number is needed with starts")
        tokens = lens.numel()
    dtype = torch.float32 if dtype is None else dtype
    pages, kv, page, batch, sp = _kv4_args(torch, cache, head_dim, tokens, table, lens, starts)
    code = _dtype_code(torch, dtype, "dtype")
    k = cache.new_empty((tokens, kv, head_dim), dtype=dtype)
    v = cache.new_empty((tokens, kv, head_dim), dtype=dtype)
    if tokens:
        st = lib().externd_kv4_read(cache.data_ptr(), pages, kv, head_dim, page, k.data_ptr(), v.data_ptr(), code,
                                    tokens, batch, sp, lens.data_ptr(), table.data_ptr(), table.shape[1],
                                    _stream_ptr(torch, stream))
        if st != OK:
            raise ExterndError(st, "externd_kv4_read")
    return k, v


def kv4_attention_workspace_bytes(heads_q: int, heads_kv: int, head_dim: int, dtype, tokens: int, batch: int,
                                  max_new: int = 1, max_len: int = 0) -> int:
    return int(lib().externd_kv4_attention_workspace_bytes(heads_q, heads_kv, head_dim,
                                                           _dtype_code(_torch(), dtype, "dtype"), tokens, batch,
                                                           max_new, max_len))


def kv4_attention_block_rows(heads_q: int, heads_kv: int, head_dim: int, dtype, tokens: int, batch: int, max_new: int = 1,
                             max_len: int = 0) -> int:
    """4 or 256: which of its two kernels ``kv4_attention`` takes (externd_kv4_attention_block_rows)."""
    return int(lib().externd_kv4_attention_block_rows(heads_q, heads_kv, head_dim, _dtype_code(_torch(), dtype, "dtype"),
                                                      tokens, batch, max_new, max_len))


def kv4_attention(cache, q, table, lens, starts=None, max_new=None, max_len=None, scale=None, window: int = 0, out=None,
                  stream=None, workspace=None):
    """Attention of the new tokens' q (tokens x query heads x channels) over
    the cache, causal, within ``window`` positions where that is above 0
    (externd_kv4_attention).  ``max_new``, ``max_len``: the most new tokens
    and the greatest length of a sequence where the caller knows them (they
    choose the launch only; without them all new tokens count as one
    sequence's, which suits prompts and not drafts of many users); ``scale``: 1 / sqrt(channels) unless given.
    Returns (out, lse): tokens x query heads x channels in q's type, and fp32
    tokens x query heads."""
    torch = _torch()
    if stream is not None:      # as on that stream: its own memory for what is allocated here
        with torch.cuda.stream(stream):
            return kv4_attention(cache, q, table, lens, starts, max_new, max_len, scale, window, out, None, workspace)
    if q.dim() != 3:
        raise ValueError(f"q: expected (tokens, heads, channels), got shape {tuple(q.shape)}")
    tokens, heads, dim = q.shape
    pages, kv, page, batch, sp = _kv4_args(torch, cache, dim, tokens, table, lens, starts)
    code = _dtype_code(torch, q.dtype, "q")
    qs = _req_heads(q, q.dtype, tokens, "q")
    if out is None:
        out = q.new_empty((tokens, heads, dim))
    else:
        _req(out, torch, q.dtype, (tokens, heads, dim), "out")
    lse = q.new_empty((tokens, heads), dtype=torch.float32)
    if not tokens:
        return out, lse
    if max_new is None:
        max_new = 1 if sp is None else tokens
    if max_len is None:
        max_len = table.shape[1] * page
    if scale is None:
        scale = dim ** -0.5
    window = min(window, 0x7FFFFFFF)      # positions are below 2^31
    L = lib()
    nbytes = L.externd_kv4_attention_workspace_bytes(heads, kv, dim, code, tokens, batch, max_new, max_len)
    wp = None
    if workspace is not None:
        if not (workspace.is_cuda and workspace.is_contiguous()):
            raise ValueError(f"workspace: expected a contiguous CUDA tensor, got {tuple(workspace.shape)} "
                             f"{workspace.stride()} on {workspace.device}")
        wp, nbytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    elif nbytes:
        workspace = cache.new_empty((nbytes,))
        wp = workspace.data_ptr()
    st = L.externd_kv4_attention(cache.data_ptr(), pages, kv, dim, page, q.data_ptr(), code, qs[0], qs[1], heads,
                                 out.data_ptr(), lse.data_ptr(), tokens, batch, max_new, max_len, sp, lens.data_ptr(),
                                 table.data_ptr(), table.shape[1], scale, window, wp, nbytes,
                                 _stream_ptr(torch, stream))
    if st != OK:
        raise ExterndError(st, "externd_kv4_attention")
    return out, lse


@dataclass
class TokenLogprobs:
    logprob: "object"          # torch.float32 (rows,): of the targets; 0 where none is asked for
    entropy: "object"          # torch.float32 (rows,)
    lse: "object"              # torch.float32 (rows,)
    top_logprobs: "object"     # torch.float32 (rows, top), the largest first; None from linear_logprobs
    top_ids: "object"          # torch.int64 (rows, top); None from linear_logprobs


def _req_logits(torch, t, name):
    if not (t.is_cuda and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1)):
        raise ValueError(f"{name}: expected a CUDA tensor (rows, vocabulary) with dense rows, got {t.dtype} "
                         f"{tuple(t.shape)} {t.stride()} on {t.device}")
    rows, vocab = t.shape
    return rows, vocab, t.stride(0) if rows > 1 else vocab, _dtype_code(torch, t.dtype, name)


def token_logprobs(logits, targets=None, top: int = 0, scale: float = 1.0, stream=None,
                   workspace=None) -> TokenLogprobs:
    """Log probabilities of the int64 ``targets`` (rows; below 0: none asked
    for) under the softmax of ``scale * logits`` (rows x vocabulary), each
    row's entropy, and its ``top`` most likely tokens, the lower index first
    among equals (externd_token_logprobs).  Without targets logprob is None.
    ``workspace`` is not used: the operator needs none."""
    torch = _torch()
    if stream is not None:      # as on that stream: its own memory for what is allocated here
        with torch.cuda.stream(stream):
            return token_logprobs(logits, targets, top, scale)
    rows, vocab, stride, code = _req_logits(torch, logits, "logits")
    if not 0 <= top <= min(LOGPROBS_MAX_TOP, vocab):
        raise ExterndError(EINVAL, "externd_token_logprobs")
    # one buffer for the three numbers of each row
    entropy, lse, logprob = logits.new_empty((3, rows), dtype=torch.float32).unbind(0)
    tp = lp = None
    if targets is not None:
        _req(targets, torch, torch.int64, (rows,), "targets")
        tp, lp = targets.data_ptr(), logprob.data_ptr()
    else:
        logprob = None
    vals = logits.new_empty((rows, top), dtype=torch.float32)
    ids = logits.new_empty((rows, top), dtype=torch.int64)
    if rows:
        st = lib().externd_token_logprobs(logits.data_ptr(), code, rows, vocab, stride, tp, scale, top, lp,
                                          entropy.data_ptr(), lse.data_ptr(), vals.data_ptr() if top else None,
                                          ids.data_ptr() if top else None, None, 0, _stream_ptr(torch, stream))
        if st != OK:
            raise ExterndError(st, "externd_token_logprobs")
    return TokenLogprobs(logprob, entropy, lse, vals, ids)


def token_logprobs_backward(logits, targets, lse, entropy, grad_logprob=None, grad_entropy=None, scale: float = 1.0,
                            out=None, stream=None):
    """Gradient for the logits from those of ``token_logprobs``'s logprob and
    entropy (externd_token_logprobs_backward); ``out`` may be the logits
    themselves.  Returns it (rows x vocabulary, the logits' type)."""
    torch = _torch()
    if stream is not None:      # as on that stream: its own memory for what is allocated here
        with torch.cuda.stream(stream):
            return token_logprobs_backward(logits, targets, lse, entropy, grad_logprob, grad_entropy, scale, out)
    rows, vocab, stride, code = _req_logits(torch, logits, "logits")
    ptrs = [None] * 5
    for i, (t, dt, name) in enumerate(((targets, torch.int64, "targets"), (lse, torch.float32, "lse"),
                                       (entropy, torch.float32, "entropy"),
                                       (grad_logprob, torch.float32, "grad_logprob"),
                                       (grad_entropy, torch.float32, "grad_entropy"))):
        if t is not None:
            _req(t, torch, dt, (rows,), name)
            ptrs[i] = t.data_ptr()
    if out is None:
        out = logits.new_empty((rows, vocab))
    orows, ovocab, ostride, _ = _req_logits(torch, out, "out")
    if (orows, ovocab) != (rows, vocab) or out.dtype is not logits.dtype:
        raise ValueError(f"out: expected {logits.dtype} of shape {(rows, vocab)}, got {out.dtype} {tuple(out.shape)}")
    if rows:
        st = lib().externd_token_logprobs_backward(logits.data_ptr(), code, rows, vocab, stride, ptrs[0], scale,
                                                   ptrs[1], ptrs[2], ptrs[3], ptrs[4], out.data_ptr(), ostride,
                                                   _stream_ptr(torch, stream))
        if st != OK:
            raise ExterndError(st, "externd_token_logprobs_backward")
    return out


# ---------------------------------------------------------------------------
# operators at a model's dense ends: the embedding, the head with the log
# probabilities behind it, and the norm of all gradients
# ---------------------------------------------------------------------------
def _given_workspace(workspace):
    """(pointer, bytes) of a workspace that the caller brings."""
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError(f"workspace: expected a contiguous CUDA tensor, got {tuple(workspace.shape)} "
                         f"{workspace.stride()} on {workspace.device}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _req_rows(torch, t, dtype, rows, width, name):
    """A CUDA matrix of dtype with dense rows; returns its row stride.  None for rows or width: any."""
    if not (t.is_cuda and t.dtype is dtype and t.dim() == 2 and (rows is None or t.shape[0] == rows)
            and (width is None or t.shape[1] == width) and (t.stride(1) == 1 or t.shape[1] == 1)):
        raise ValueError(f"{name}: expected a {dtype} CUDA tensor ({'rows' if rows is None else rows}, "
                         f"{'width' if width is None else width}) with dense rows, got {t.dtype} {tuple(t.shape)} "
                         f"{t.stride()} on {t.device}")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _overlaps(a, b) -> bool:
    """Whether two matrices with dense rows have bytes in common."""
    if not a.numel() or not b.numel():
        return False
    size, (a0, b0) = a.element_size(), (a.data_ptr(), b.data_ptr())
    wa, wb = a.shape[1] * size, b.shape[1] * size
    sa, sb = (t.stride(0) * size if t.shape[0] > 1 else None for t in (a, b))      # None: a single row, at any distance from the next
    sa, sb = sa or sb or wa, sb or sa or wb
    if a0 >= b0 + (b.shape[0] - 1) * sb + wb or b0 >= a0 + (a.shape[0] - 1) * sa + wa:
        return False
    return not (sa == sb > 0 and (b0 - a0) % sa >= wa and (b0 - a0) % sa + wb <= sa)      # columns side by side in one buffer


def _elsewhere(torch, t, stream):
    """Where the call has to be made again: on the given stream (with its own
    memory for what is allocated) or on the device of t; None: here."""
    if stream is not None:
        if stream.device != t.device:
            raise ValueError(f"stream: on {stream.device}, the tensors on {t.device}")
        return torch.cuda.stream(stream)
    if t.is_cuda and t.device.index != torch.cuda.current_device():
        return torch.cuda.device(t.device)
    return None


def _same_device(t, *others):
    for o in others:
        if o is not None and o.device != t.device:
            raise ValueError(f"all tensors must be on one device, got {t.device} and {o.device}")


def embedding(table, ids, scale: float = 1.0, out=None, stream=None):
    """``scale * table[ids]`` (externd_embedding): table (vocabulary x width),
    ids int64 of any shape, in a row; one outside the vocabulary (padding) gives
    zeros.  Returns ids.shape + (width,) in the table's type, or ``out`` (tokens
    x width, dense rows)."""
    torch = _torch()
    there = _elsewhere(torch, table, stream)
    if there is not None:
        with there:
            return embedding(table, ids, scale, out)
    code = _dtype_code(torch, table.dtype, "table")
    stride = _req_rows(torch, table, table.dtype, None, None, "table")
    vocab, width = table.shape
    _req(ids, torch, torch.int64, ids.shape, "ids")
    _same_device(table, ids, out)
    tokens = ids.numel()
    if out is None:
        got = table.new_empty((*ids.shape, width))
        ostride = width
    else:
        got = out
        ostride = _req_rows(torch, out, table.dtype, tokens, width, "out")
        if _overlaps(out, table):
            raise ValueError("out: must not overlap the table")
    st = lib().externd_embedding(table.data_ptr(), code, vocab, width, stride, ids.data_ptr(), tokens, scale, got.data_ptr(),
                                 ostride, _stream_ptr(torch, stream))
    if st != OK:
        raise ExterndError(st, "externd_embedding")
    return got


def embedding_backward(grad, ids, vocab: int, scale: float = 1.0, out=None, accumulate: bool = False, stream=None,
                       workspace=None):
    """Gradient of ``embedding`` for the table (externd_embedding_backward):
    grad (ids.shape + (width,), dense rows) summed over each id's places, times
    scale.  ``out`` (vocab x width): where it goes; with ``accumulate`` it is
    added to what ``out`` holds, as where head and embedding are one matrix.
    Bit-identical from run to run.  Returns (vocab x width)."""
    torch = _torch()
    there = _elsewhere(torch, grad, stream)
    if there is not None:
        with there:
            return embedding_backward(grad, ids, vocab, scale, out, accumulate, None, workspace)
    code = _dtype_code(torch, grad.dtype, "grad")
    _req(ids, torch, torch.int64, ids.shape, "ids")
    if grad.dim() < 1 or grad.shape[:-1] != ids.shape:
        raise ValueError(f"grad: expected shape {tuple(ids.shape)} + (width,), got {tuple(grad.shape)}")
    width, tokens = grad.shape[-1], ids.numel()
    if grad.dim() != 2:
        if not grad.is_contiguous():
            raise ValueError(f"grad: more or fewer than two dimensions must be contiguous, got strides {grad.stride()}")
        grad = grad.view(tokens, width)
    gstride = _req_rows(torch, grad, grad.dtype, tokens, width, "grad")
    if out is None:
        if accumulate:
            raise ValueError("out: needed to accumulate into")
        out = grad.new_empty((vocab, width))
    ostride = _req_rows(torch, out, grad.dtype, vocab, width, "out")
    _same_device(grad, ids, out, workspace)
    if _overlaps(out, grad):
        raise ValueError("out: must not overlap grad")
    L = lib()
    nbytes = L.externd_embedding_backward_workspace_bytes(tokens, vocab, width)
    wp = None
    if workspace is not None:
        wp, nbytes = _given_workspace(workspace)
    elif nbytes:
        workspace = grad.new_empty((nbytes,), dtype=torch.uint8)
        wp = workspace.data_ptr()
    st = L.externd_embedding_backward(grad.data_ptr(), code, tokens, width, gstride, ids.data_ptr(), vocab, scale,
                                      int(accumulate), out.data_ptr(), ostride, wp, nbytes, _stream_ptr(torch, stream))
    if st != OK:
        raise ExterndError(st, "externd_embedding_backward")
    return out


def linear_logprobs(x, weight, targets=None, scale: float = 1.0, stream=None, workspace=None) -> TokenLogprobs:
    """``token_logprobs`` of the logits ``x weight^T`` (x: rows x width, weight:
    vocabulary x width, of one type), which are never held
    (externd_linear_logprobs): log probabilities of the int64 ``targets``, entropies
    and lse.  The largest logits are not kept: the top fields are None, and
    without targets logprob is."""
    torch = _torch()
    there = _elsewhere(torch, x, stream)
    if there is not None:
        with there:
            return linear_logprobs(x, weight, targets, scale, None, workspace)
    code = _dtype_code(torch, x.dtype, "x")
    xs = _req_rows(torch, x, x.dtype, None, None, "x")
    rows, width = x.shape
    ws = _req_rows(torch, weight, x.dtype, None, width, "weight")
    vocab = weight.shape[0]
    _same_device(x, weight, targets, workspace)
    entropy, lse, logprob = x.new_empty((3, rows), dtype=torch.float32).unbind(0)
    tp = lp = None
    if targets is not None:
        _req(targets, torch, torch.int64, (rows,), "targets")
        tp, lp = targets.data_ptr(), logprob.data_ptr()
    else:
        logprob = None
    L = lib()
    wp, nbytes = None, 0
    if workspace is not None:
        wp, nbytes = _given_workspace(workspace)
    elif rows:
        nbytes = L.externd_linear_logprobs_workspace_bytes(code, rows, vocab, width)
        workspace = x.new_empty((nbytes,), dtype=torch.uint8)
        wp = workspace.data_ptr()
    st = L.externd_linear_logprobs(x.data_ptr(), xs, weight.data_ptr(), ws, code, rows, vocab, width, tp, scale, lp,
                                   entropy.data_ptr(), lse.data_ptr(), wp, nbytes, _stream_ptr(torch, stream))
    if st != OK:
        raise ExterndError(st, "externd_linear_logprobs")
    return TokenLogprobs(logprob, entropy, lse, None, None)


def linear_logprobs_backward(x, weight, targets, lse, entropy, grad_logprob=None, grad_entropy=None, scale: float = 1.0,
                             need_x: bool = True, need_weight: bool = True, out=None, stream=None, workspace=None):
    """Gradients for x and weight from those of ``linear_logprobs``'s logprob
    and entropy (externd_linear_logprobs_backward), with its lse and entropy.
    ``need_x``, ``need_weight``: which are asked for; ``out``: (grad_x,
    grad_weight), where they go.  Rows whose two gradients are 0 (padding) take no
    part, whatever x holds there.  Returns (grad_x, grad_weight), None for what
    is not asked for."""
    torch = _torch()
    there = _elsewhere(torch, x, stream)
    if there is not None:
        with there:
            return linear_logprobs_backward(x, weight, targets, lse, entropy, grad_logprob, grad_entropy, scale, need_x,
                                            need_weight, out, None, workspace)
    code = _dtype_code(torch, x.dtype, "x")
    xs = _req_rows(torch, x, x.dtype, None, None, "x")
    rows, width = x.shape
    ws = _req_rows(torch, weight, x.dtype, None, width, "weight")
    vocab = weight.shape[0]
    ptrs = [None] * 5
    for i, (t, dt, name) in enumerate(((targets, torch.int64, "targets"), (lse, torch.float32, "lse"),
                                       (entropy, torch.float32, "entropy"),
                                       (grad_logprob, torch.float32, "grad_logprob"),
                                       (grad_entropy, torch.float32, "grad_entropy"))):
        if t is not None:
            _req(t, torch, dt, (rows,), name)
            ptrs[i] = t.data_ptr()
    gx, gw = out if out is not None else (None, None)
    gx = (x.new_empty((rows, width)) if gx is None else gx) if need_x else None
    gw = (x.new_empty((vocab, width)) if gw is None else gw) if need_weight else None
    gxs = _req_rows(torch, gx, x.dtype, rows, width, "grad_x") if need_x else width
    gws = _req_rows(torch, gw, x.dtype, vocab, width, "grad_weight") if need_weight else width
    _same_device(x, weight, targets, lse, entropy, grad_logprob, grad_entropy, gx, gw, workspace)
    outs = [t for t in (gx, gw) if t is not None]
    if any(_overlaps(o, t) for o in outs for t in (x, weight)) or (len(outs) == 2 and _overlaps(*outs)):
        raise ValueError("out: must overlap neither x nor weight nor each other")
    if not outs:
        return None, None
    L = lib()
    if workspace is not None:
        wp, nbytes = _given_workspace(workspace)
    else:
        nbytes = L.externd_linear_logprobs_backward_workspace_bytes(code, rows, vocab, width, int(need_x), int(need_weight))
        workspace = x.new_empty((nbytes,), dtype=torch.uint8)
        wp = workspace.data_ptr()
    st = L.externd_linear_logprobs_backward(x.data_ptr(), xs, weight.data_ptr(), ws, code, rows, vocab, width, ptrs[0], scale,
                                            ptrs[1], ptrs[2], ptrs[3], ptrs[4], gx.data_ptr() if need_x else None, gxs,
                                            gw.data_ptr() if need_weight else None, gws, wp, nbytes,
                                            _stream_ptr(torch, stream))
    if st != OK:
        raise ExterndError(st, "externd_linear_logprobs_backward")
    return gx, gw


def _dense(t) -> bool:
    """Whether t's entries fill its memory without gaps, in any order of the dimensions."""
    if t.is_contiguous():
        return True
    want = 1
    for n, s in sorted(((n, s) for n, s in zip(t.shape, t.stride()) if n > 1), key=lambda d: d[1]):
        if s != want:
            return False
        want *= n
    return True


def _written_twice(ins, ops, nbytes) -> bool:
    """Whether an output's memory has bytes in common with another output, or with
    an input that is not its own (inputs may share theirs: they are only read)."""
    if len(ins) <= 32:
        spans = [(o, o + n, True) for o, n in zip(ops, nbytes) if n]
        if ops is not ins:
            spans += [(i, i + n, False) for i, o, n in zip(ins, ops, nbytes) if n and i != o]
        spans.sort()
        end = end_wrote = 0
        for a, b, wrote in spans:
            if a < end_wrote or (wrote and a < end):
                return True
            end = max(end, b)
            end_wrote = max(end_wrote, b) if wrote else end_wrote
        return False
    a, size = np.asarray(ops, dtype=np.int64), np.asarray(nbytes, dtype=np.int64)      # the same without a loop
    keep, wrote = size > 0, np.ones(len(ops), dtype=bool)
    if ops is not ins:
        i = np.asarray(ins, dtype=np.int64)
        keep = np.concatenate([keep, keep & (i != a)])
        a, size, wrote = np.concatenate([a, i]), np.concatenate([size, size]), np.concatenate([wrote, ~wrote])
    a, size, wrote = a[keep], size[keep], wrote[keep]
    order = np.argsort(a, kind="stable")
    a, b, wrote = a[order], (a + size)[order], wrote[order]
    end, end_wrote = np.maximum.accumulate(b), np.maximum.accumulate(np.where(wrote, b, 0))
    return bool(np.any((a[1:] < end[:-1]) & wrote[1:]) or np.any(a[1:] < end_wrote[:-1]))


def clip_gradients(tensors, max_norm: float = float("inf"), out=None, stream=None, workspace=None):
    """The norm over all entries of ``tensors`` (CUDA, dense, float32, bfloat16
    or float16, mixed), and each of them times min(1, max_norm / norm), in place
    or into ``out`` (as many tensors of the same sizes and types, and of the same
    strides where they are not contiguous) (externd_clip_gradients).  With max_norm infinite only the norm.  Returns
    the norm, a float32 CUDA scalar; nothing is copied to the host."""
    torch = _torch()
    tensors = list(tensors)
    if tensors or stream is not None:
        there = _elsewhere(torch, tensors[0] if tensors else stream, stream)
        if there is not None:
            with there:
                return clip_gradients(tensors, max_norm, out, None, workspace)
    outs = tensors if out is None else list(out)
    if len(outs) != len(tensors):
        raise ValueError(f"out: expected {len(tensors)} tensors, got {len(outs)}")
    if not max_norm >= 0:
        raise ExterndError(EINVAL, "externd_clip_gradients")
    device = tensors[0].device if tensors else torch.device("cuda", torch.cuda.current_device())
    index = device.index
    if workspace is not None and workspace.device != device:
        raise ValueError(f"workspace: expected on {device}, got {workspace.device}")
    if _dtype_codes is None:
        _dtype_code(torch, torch.float32, "")
    # hundreds of tensors are ordinary, so each property is taken of all at once (216
    # and as many outputs: 180 us a call, nearly all of it here, -> 141)
    T = torch.Tensor
    dtypes = [t.dtype for t in tensors]
    codes = list(map(_dtype_codes.get, dtypes))
    gaps = False in map(T.is_contiguous, tensors)
    if None in codes or not {index}.issuperset(map(T.get_device, tensors)) or (gaps and not all(map(_dense, tensors))):
        i = next(i for i, t in enumerate(tensors) if t.dtype not in _dtype_codes or t.get_device() != index or not _dense(t))
        t = tensors[i]
        raise ValueError(f"tensors[{i}]: expected a dense CUDA tensor of float32, bfloat16 or float16 on {device}, got "
                         f"{t.dtype} {tuple(t.shape)} {t.stride()} on {t.device}")
    ops = ins = list(map(T.data_ptr, tensors))
    sizes = list(map(T.numel, tensors))
    if out is not None:
        if (gaps or False in map(T.is_contiguous, outs) or [o.dtype for o in outs] != dtypes
                or list(map(T.numel, outs)) != sizes or not {index}.issuperset(map(T.get_device, outs))):
            for i, (t, o) in enumerate(zip(tensors, outs)):
                if not (o.dtype is t.dtype and o.get_device() == index and o.shape == t.shape
                        and (o.is_contiguous() and t.is_contiguous() or o.stride() == t.stride())):
                    raise ValueError(f"out[{i}]: expected {t.dtype} {tuple(t.shape)} {t.stride()} on {t.device}, got {o.dtype} "
                                     f"{tuple(o.shape)} {o.stride()} on {o.device}")
        ops = list(map(T.data_ptr, outs))
    n = len(tensors)
    counts, types = np.array(sizes, dtype=np.int64), np.array(codes, dtype=np.int32)
    in_ptrs = np.array(ins, dtype=np.int64)
    out_ptrs = in_ptrs if ops is ins else np.array(ops, dtype=np.int64)
    if max_norm != float("inf") and tensors:
        if n <= 32:
            twice = _written_twice(ins, ops, [m * (4 if c == 0 else 2) for m, c in zip(sizes, codes)])
        else:
            twice = _written_twice(in_ptrs, out_ptrs, counts << (1 + (types == 0)))
        if twice:
            raise ValueError("tensors: what is written overlaps another tensor")
    norm = torch.empty((), dtype=torch.float32, device=device)
    L = lib()
    if workspace is not None:
        wp, nbytes = _given_workspace(workspace)
    else:
        nbytes = L.externd_clip_gradients_workspace_bytes(n)
        workspace = torch.empty((nbytes,), dtype=torch.uint8, device=device)
        wp = workspace.data_ptr()
    st = L.externd_clip_gradients(n, in_ptrs.ctypes.data, None if ops is ins else out_ptrs.ctypes.data, counts.ctypes.data,
                                  types.ctypes.data, max_norm, norm.data_ptr(), wp, nbytes, _stream_ptr(torch, stream))
    if st != OK:
        raise ExterndError(st, "externd_clip_gradients")
    return norm


# ---------------------------------------------------------------------------
# packed trit format (host-side decode for users and tests)
# ---------------------------------------------------------------------------
def unpack_trits(packed: np.ndarray, cols: int) -> np.ndarray:
    """Decode rows of 2-bit trits (00 = 0, 01 = +1, 11 = -1) into int8.

    Raises ValueError on the unused code 10 or on nonzero padding bits.
    """
    packed = np.ascontiguousarray(packed, dtype=np.uint8)
    rows, nbytes = packed.shape
    if nbytes != (cols + 3) // 4:
        raise ValueError("packed row length does not match the column count")
    codes = np.stack([(packed >> (2 * s)) & 3 for s in range(4)], axis=-1).reshape(rows, nbytes * 4)
    if np.any(codes == 2):
        raise ValueError("invalid trit code 10")
    if np.any(codes[:, cols:] != 0):
        raise ValueError("nonzero padding bits")
    codes = codes[:, :cols]
    out = np.zeros((rows, cols), dtype=np.int8)
    out[codes == 1] = 1
    out[codes == 3] = -1
    return out
