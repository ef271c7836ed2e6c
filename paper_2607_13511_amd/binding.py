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
    top_logprobs: "object"     # torch.float32 (rows, top), the largest first
    top_ids: "object"          # torch.int64 (rows, top)


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
