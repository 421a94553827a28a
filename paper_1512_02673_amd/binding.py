"""ctypes binding of libcoded_mi355x.so: the C ABI's calls under the same names.

Argument marshalling only: shapes, strides and data pointers are read from
torch tensors, the current torch stream is passed as the HIP stream, and every
step of the coded product runs in the library.  Loading fails loudly when the
library has not been built.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
import re

import numpy as np

from .build import LIB_PATH

CODED_OK, CODED_ERR_ARG, CODED_ERR_SHAPE, CODED_ERR_TOO_FEW, CODED_ERR_SINGULAR, CODED_ERR_HIP, \
    CODED_ERR_UNSUPPORTED = range(7)
CODED_F32, CODED_BF16, CODED_F64, CODED_MX4, CODED_MX8 = 0, 1, 2, 3, 4
CODED_X_ROWS, CODED_Y_ROWS = 1, 2
CODED_MAX_N = 128
CODED_NOALLOC_SCRATCH_BYTES = 64 << 20
CODED_PLANES_LO_BF16 = 3   # fp32 codes: hi plane fp32, lo plane bfloat16

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "coded.h")

_c_i32, _c_i64, _c_u64, _c_dbl, _c_p = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_double, ctypes.c_void_p

_SIGNATURES = {
    "coded_code_bytes": (_c_i32, [_c_i32, _c_i32, _c_p]),
    "coded_code_create": (_c_i32, [_c_i32, _c_i32, _c_p, _c_i32, _c_p, _c_i64, ctypes.POINTER(_c_p)]),
    "coded_code_destroy": (_c_i32, [_c_p]),
    "coded_code_info": (_c_i32, [_c_p, _c_p, _c_p, _c_p]),
    "coded_sizes": (_c_i32, [_c_p, _c_i32, _c_i32, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p]),
    "coded_encode": (_c_i32, [_c_p, _c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p]),
    "coded_worker_mm": (_c_i32, [_c_p, _c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_i64, _c_i64, _c_p,
                                 _c_p, _c_i32, _c_p, _c_p]),
    "coded_encode_worker_mm": (_c_i32, [_c_p, _c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_i64, _c_i64,
                                        _c_p, _c_i32, _c_p, _c_p]),
    "coded_decode": (_c_i32, [_c_p, _c_p, _c_i32, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_i64, _c_p, _c_p]),
    "coded_decode_batched": (_c_i32, [_c_p, _c_p, _c_i32, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_i64, _c_i64,
                                      _c_p, _c_p]),
    "coded_draw_survivors": (_c_i32, [_c_i32, _c_i32, _c_u64, _c_u64, _c_dbl, _c_dbl, _c_p, _c_p]),
    "coded_draw_survivor_sets": (_c_i32, [_c_i32, _c_i32, _c_u64, _c_u64, _c_i32, _c_i32, _c_p, _c_p]),
    "coded_matmul": (_c_i32, [_c_p, _c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i32, _c_p, _c_i64, _c_i64,
                              _c_u64, _c_u64, _c_dbl, _c_dbl, _c_p, _c_p, _c_p, _c_i64, _c_p, _c_p, _c_p]),
    "coded_matmul_noalloc": (_c_i32, [_c_p, _c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i32, _c_p, _c_i64, _c_i64,
                                      _c_u64, _c_u64, _c_dbl, _c_dbl, _c_p, _c_p, _c_p, _c_i64, _c_p, _c_p]),
    "coded_straggler_matmul": (_c_i32, [_c_p, _c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_i64, _c_i64,
                                        _c_u64, _c_u64, _c_dbl, _c_dbl, _c_dbl, _c_i32, _c_p, _c_i32, _c_p, _c_p,
                                        _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "coded_transpose": (_c_i32, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i64, _c_p]),
    "coded_shuffle_create": (_c_i32, [_c_i32, _c_i64, _c_i64, _c_u64, _c_p]),
    "coded_shuffle_destroy": (_c_i32, [_c_p]),
    "coded_shuffle_state": (_c_i32, [_c_p, _c_p, _c_p, _c_p]),
    "coded_shuffle_plan": (_c_i32, [_c_p, _c_p, _c_p]),
    "coded_shuffle_tables": (_c_i32, [_c_p, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "coded_shuffle_commit": (_c_i32, [_c_p]),
    "coded_shuffle_encode": (_c_i32, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_i64, _c_i64, _c_p, _c_i64, _c_p]),
    "coded_shuffle_decode": (_c_i32, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i64, _c_p, _c_p, _c_p, _c_i64, _c_i64,
                                      _c_p, _c_i64, _c_p]),
    "coded_gd_sizes": (_c_i32, [_c_p, _c_p, _c_i64, _c_i64, _c_p]),
    "coded_gd_step": (_c_i32, [_c_p, _c_p, _c_p, _c_i64, _c_p, _c_p, _c_i64, _c_p, _c_i64, _c_i64, _c_p, _c_p, _c_dbl,
                               _c_u64, _c_u64, _c_dbl, _c_dbl, _c_p, _c_p, _c_p, _c_p]),
    "coded_simulate_runtimes": (_c_i32, [_c_i32, _c_i32, _c_u64, _c_u64, _c_i64, _c_dbl, _c_dbl, _c_p, _c_p, _c_p,
                                         _c_p]),
    "coded_optimal_k": (_c_i32, [_c_i32, _c_dbl, _c_p, _c_p, _c_p]),
    "coded_mx_sizes": (_c_i32, [_c_i32, _c_i64, _c_p, _c_p]),
    "coded_mx_quantize": (_c_i32, [_c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_i32, _c_p, _c_i64, _c_p, _c_i64, _c_p]),
    "coded_mx_dequantize": (_c_i32, [_c_i32, _c_p, _c_i64, _c_p, _c_i64, _c_i64, _c_i64, _c_i32, _c_p, _c_i64, _c_p]),
    "coded_mx_workspace": (_c_i32, [_c_i32, _c_i32, _c_i64, _c_i64, _c_i32, _c_i64, _c_i32, _c_p]),
    "coded_mx_mm": (_c_i32, [_c_i32, _c_p, _c_i64, _c_p, _c_i64, _c_i64, _c_i64, _c_i32, _c_p, _c_i64, _c_p, _c_i64,
                             _c_i64, _c_i32, _c_dbl, _c_dbl, _c_p, _c_i64, _c_p, _c_i32, _c_i64, _c_p, _c_i64, _c_p]),
    "coded_mx_mm_t": (_c_i32, [_c_i32, _c_p, _c_i64, _c_p, _c_i64, _c_i64, _c_i64, _c_i32, _c_p, _c_i64, _c_i64,
                               _c_i32, _c_dbl, _c_dbl, _c_p, _c_i64, _c_p, _c_i32, _c_i64, _c_p, _c_i64, _c_p]),
    "coded_f8_sizes": (_c_i32, [_c_i64, _c_i64, _c_i32, _c_p, _c_p]),
    "coded_f8_quantize": (_c_i32, [_c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_i32, _c_p, _c_i64, _c_p, _c_i64, _c_i32, _c_p,
                                   _c_i64, _c_p, _c_i64, _c_p]),
    "coded_f8_dequantize": (_c_i32, [_c_i64, _c_i64, _c_i32, _c_p, _c_i64, _c_p, _c_i64, _c_i32, _c_p, _c_i64, _c_p]),
    "coded_f8_workspace": (_c_i32, [_c_i64, _c_i64, _c_i64, _c_i32, _c_i32, _c_p]),
    "coded_f8_mm": (_c_i32, [_c_i64, _c_i64, _c_i64, _c_i32, _c_p, _c_i64, _c_p, _c_i64, _c_i32, _c_p, _c_i64, _c_p, _c_i64,
                             _c_i32, _c_dbl, _c_dbl, _c_p, _c_i64, _c_p, _c_i32, _c_i64, _c_p, _c_i64, _c_p]),
    "coded_dropout": (_c_i32, [_c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_dbl, _c_u64, _c_u64, _c_i64, _c_p, _c_i64, _c_p, _c_i64,
                               _c_p]),
    "coded_embed": (_c_i32, [_c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i32, _c_i64, _c_i64, _c_dbl, _c_i32, _c_p, _c_i64,
                             _c_p]),
    "coded_embed_workspace": (_c_i32, [_c_i64, _c_i64, _c_i64, _c_p]),
    "coded_embed_grad": (_c_i32, [_c_i32, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_i32, _c_i64, _c_i64, _c_dbl, _c_dbl, _c_i32,
                                  _c_p, _c_i64, _c_p, _c_i64, _c_p]),
    "coded_status_string": (ctypes.c_char_p, [_c_i32]),
    "coded_last_error": (ctypes.c_char_p, []),
    "coded_version": (ctypes.c_char_p, []),
}

_lib = None


class CodedError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{status_string(status)}: {message}")
        self.status = status


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it is not built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built: run paper_1512_02673_amd.build.build() "
                               "(or __graft_entry__.build()) first")
        h = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            f = getattr(h, name)
            f.restype = res
            f.argtypes = args
        _lib = h
    return _lib


def header_functions() -> list[str]:
    """Names of the functions include/coded.h declares."""
    text = open(HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(coded_[a-z0-9_]+)\s*\(", text)))


def status_string(status: int) -> str:
    return lib().coded_status_string(status).decode()


def last_error() -> str:
    return lib().coded_last_error().decode()


def version() -> str:
    return lib().coded_version().decode()


def _check(status: int) -> None:
    if status != CODED_OK:
        raise CodedError(status, last_error())


# ---------------------------------------------------------------- host-only calls

def coded_draw_survivors(n: int, k: int, seed: int, draw: int, shift: float = 1.0, rate: float = 1.0):
    """(survivors ascending int32[k], T_(k)) of one draw."""
    out = np.zeros(k, dtype=np.int32)
    t = ctypes.c_double()
    _check(lib().coded_draw_survivors(n, k, seed, draw, shift, rate, out.ctypes.data, ctypes.addressof(t)))
    return out, t.value


def coded_draw_survivor_sets(n: int, k: int, seed: int, batch: int, min_parity: int = 0, first_draw: int = 0):
    """(sets int32[batch, k], next unused draw)."""
    out = np.zeros((batch, k), dtype=np.int32)
    nxt = ctypes.c_uint64()
    _check(lib().coded_draw_survivor_sets(n, k, seed, first_draw, batch, min_parity, out.ctypes.data,
                                          ctypes.addressof(nxt)))
    return out, nxt.value


def coded_optimal_k(n: int, rate: float):
    """(k*, T*, best integer k) of Lemma 2."""
    ks, ts, kb = ctypes.c_double(), ctypes.c_double(), ctypes.c_int32()
    _check(lib().coded_optimal_k(n, rate, ctypes.addressof(ks), ctypes.addressof(ts), ctypes.addressof(kb)))
    return ks.value, ts.value, kb.value


# ---------------------------------------------------------------- device calls

def _torch():
    import torch
    return torch


def _stream(stream=None):
    """The HIP stream handle of `stream`, or of the current device's current stream, read
    without making a Stream object (3 us of a small call's 12) where torch has the call for it,
    which is not part of its public interface."""
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device())


def _memory_of(stream):
    """Within it torch hands out memory of `stream` (None: the current one): memory of the current
    stream's may still be in use by what waits there, and another stream does not wait for that."""
    return contextlib.nullcontext() if stream is None else _torch().cuda.stream(stream)


def _given(workspace):
    """(data, bytes) of a caller's workspace.  The elements of an expanded one are more than its memory holds."""
    if not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


_DTYPE_CODES: dict = {}   # filled on first use: torch is imported late


def _dtype_code(t) -> int:
    if not _DTYPE_CODES:
        torch = _torch()
        _DTYPE_CODES.update({torch.float32: CODED_F32, torch.bfloat16: CODED_BF16, torch.float64: CODED_F64})
    return _DTYPE_CODES[t.dtype]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _matrix(t, name):
    """(rows, cols, row stride) of a 1-D (column) or row-major 2-D tensor."""
    if t.dim() == 1:
        if t.stride(0) != 1:
            raise ValueError(f"{name} must be contiguous")
        return t.shape[0], 1, 1
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name} must be 1-D or row-major 2-D")
    return t.shape[0], t.shape[1], max(t.stride(0), 1)


def coded_code_bytes(n: int, k: int) -> int:
    """Bytes of the device buffer an (n,k) code needs."""
    b = ctypes.c_int64()
    _check(lib().coded_code_bytes(n, k, ctypes.addressof(b)))
    return b.value


class Code:
    """An (n,k) code: G = [I_k; P] on host, and on the device in a buffer this
    object owns (a torch tensor on the current device) and passes to
    coded_code_create."""

    def __init__(self, n: int, k: int, G: np.ndarray, planes: int = 2):
        G = np.ascontiguousarray(G, dtype=np.float64)
        if G.shape != (n, k):
            raise ValueError("G must be n x k")
        nbytes = coded_code_bytes(n, k)
        self.device_buf = _torch().empty(nbytes, dtype=_torch().uint8, device="cuda")
        h = ctypes.c_void_p()
        _check(lib().coded_code_create(n, k, G.ctypes.data, planes, ctypes.c_void_p(self.device_buf.data_ptr()),
                                       nbytes, ctypes.byref(h)))
        self.handle = h
        self.n, self.k, self.planes = n, k, planes
        self.G = G

    @classmethod
    def systematic(cls, P: np.ndarray, planes: int = 2) -> "Code":
        P = np.asarray(P, dtype=np.float64)
        k = P.shape[1]
        return cls(k + P.shape[0], k, np.vstack([np.eye(k), P]), planes)

    def qb(self, q: int) -> int:
        return -(-q // self.k)

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            lib().coded_code_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def coded_sizes(code: Code, dt: int, y_dt: int, q: int, r: int, s: int):
    """(parity_bytes, y_bytes, matmul workspace_bytes, worker workspace_bytes)."""
    pb, yb, wb, ww = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    _check(lib().coded_sizes(code.handle, dt, y_dt, q, r, s, ctypes.addressof(pb), ctypes.addressof(yb),
                             ctypes.addressof(wb), ctypes.addressof(ww)))
    return pb.value, yb.value, wb.value, ww.value


def coded_encode(code: Code, A, parity, stream=None) -> None:
    q, r, lda = _matrix(A, "A")
    _check(lib().coded_encode(code.handle, _dtype_code(A), _ptr(A), q, r, lda, _ptr(parity), _stream(stream)))


def worker_workspace(code: Code, A, X):
    """A device buffer of the worker workspace size for these operands (None if 0 bytes)."""
    torch = _torch()
    q, r, _ = _matrix(A, "A")
    _, s, _ = _matrix(X, "X")
    y_dt = CODED_F32 if _dtype_code(A) == CODED_BF16 else CODED_F64
    nbytes = coded_sizes(code, _dtype_code(A), y_dt, q, r, s)[3]
    return torch.empty(nbytes, dtype=torch.uint8, device=A.device) if nbytes else None


def matmul_workspace(code: Code, A, X):
    """A device buffer of coded_matmul's workspace size for these operands."""
    torch = _torch()
    q, r, _ = _matrix(A, "A")
    _, s, _ = _matrix(X, "X")
    y_dt = CODED_F32 if _dtype_code(A) == CODED_BF16 else CODED_F64
    nbytes = coded_sizes(code, _dtype_code(A), y_dt, q, r, s)[2]
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=A.device)


def coded_worker_mm(code: Code, A, parity, X, Y, worker_mask=None, workspace="auto", stream=None) -> None:
    """workspace: not used by the products; None, "auto", or a device buffer of coded_sizes'
    worker workspace bytes."""
    q, r, lda = _matrix(A, "A")
    rx, s, ldx = _matrix(X, "X")
    if rx != r:
        raise ValueError("X must have r rows")
    mask = None
    if worker_mask is not None:
        m = np.ascontiguousarray(worker_mask, dtype=np.uint8)
        if m.shape != (code.n,):
            raise ValueError("worker_mask must have n entries")
        mask = m.ctypes.data
    if isinstance(workspace, str):
        workspace = None
    _check(lib().coded_worker_mm(code.handle, _dtype_code(A), _ptr(A), q, r, lda, _ptr(parity), _ptr(X), s, ldx,
                                 mask, _ptr(Y), _dtype_code(Y), _ptr(workspace), _stream(stream)))


def coded_encode_worker_mm(code: Code, A, parity, X, Y, workspace="auto", stream=None) -> None:
    """Parity blocks and every worker's product in one call (coded_encode, then
    coded_worker_mm for all workers; one pass over A where the kernel serves the shape)."""
    q, r, lda = _matrix(A, "A")
    rx, s, ldx = _matrix(X, "X")
    if rx != r:
        raise ValueError("X must have r rows")
    if isinstance(workspace, str):
        with _memory_of(stream):
            workspace = worker_workspace(code, A, X)
    _check(lib().coded_encode_worker_mm(code.handle, _dtype_code(A), _ptr(A), q, r, lda, _ptr(parity), _ptr(X), s,
                                        ldx, _ptr(Y), _dtype_code(Y), _ptr(workspace), _stream(stream)))


def coded_decode(code: Code, survivors, Y, q: int, out, info, stream=None) -> None:
    sv = np.ascontiguousarray(survivors, dtype=np.int32)
    _, s, ldo = _matrix(out, "out")
    _check(lib().coded_decode(code.handle, sv.ctypes.data, len(sv), _ptr(Y), _dtype_code(Y), q,
                              s, _ptr(out), ldo, _ptr(info), _stream(stream)))


def coded_decode_batched(code: Code, sets, Y, q: int, out, info, stream=None) -> None:
    """sets: device int32 (batch, k); out: (batch, q) or (batch, q, s) float32."""
    batch = sets.shape[0]
    if out.dim() == 2:
        s, ldo = 1, 1
    else:
        s, ldo = out.shape[2], out.stride(1)
    _check(lib().coded_decode_batched(code.handle, _ptr(sets), batch, _ptr(Y), _dtype_code(Y), q, s, _ptr(out), ldo,
                                      out.stride(0), _ptr(info), _stream(stream)))


def coded_matmul(code: Code, A, parity, X, out, workspace, info, seed: int, draw: int, parity_ready: bool = True,
                 shift: float = 1.0, rate: float = 1.0, stream=None):
    """One coded product; returns (survivors int32[k], T_(k))."""
    q, r, lda = _matrix(A, "A")
    rx, s, ldx = _matrix(X, "X")
    if rx != r:
        raise ValueError("X must have r rows")
    _, so, ldo = _matrix(out, "out")
    surv = np.zeros(code.k, dtype=np.int32)
    t = ctypes.c_double()
    _check(lib().coded_matmul(code.handle, _dtype_code(A), _ptr(A), q, r, lda, _ptr(parity), int(bool(parity_ready)),
                              _ptr(X), s, ldx, seed, draw, shift, rate, surv.ctypes.data,
                              ctypes.addressof(t), _ptr(out), ldo, _ptr(workspace), _ptr(info), _stream(stream)))
    return surv, t.value


def coded_matmul_noalloc(code: Code, A, parity, X, out, info, seed: int, draw: int, parity_ready: bool = True,
                         shift: float = 1.0, rate: float = 1.0, stream=None):
    """coded_matmul on the library's static device scratch (no workspace argument,
    nothing allocated); returns (survivors int32[k], T_(k))."""
    q, r, lda = _matrix(A, "A")
    rx, s, ldx = _matrix(X, "X")
    if rx != r:
        raise ValueError("X must have r rows")
    _, so, ldo = _matrix(out, "out")
    surv = np.zeros(code.k, dtype=np.int32)
    t = ctypes.c_double()
    _check(lib().coded_matmul_noalloc(code.handle, _dtype_code(A), _ptr(A), q, r, lda, _ptr(parity),
                                      int(bool(parity_ready)), _ptr(X), s, ldx, seed, draw, shift, rate,
                                      surv.ctypes.data, ctypes.addressof(t), _ptr(out), ldo,
                                      _ptr(info), _stream(stream)))
    return surv, t.value


def coded_straggler_matmul(code: Code, A, parity, X, Y, out, info, seed: int, draw: int, time_unit_us: float,
                           launch_all: bool = False, workspace="auto", shift: float = 1.0, rate: float = 1.0,
                           stream=None):
    """One coded product with real, timed straggling (blocks until the decode is done).
    Returns (survivors int32[k] in arrival order, timeline float64[n, 3] in microseconds:
    start time, enqueue time, completion seen, -1 where it did not happen, latency in microseconds)."""
    q, r, lda = _matrix(A, "A")
    rx, s, ldx = _matrix(X, "X")
    if rx != r:
        raise ValueError("X must have r rows")
    _, so, ldo = _matrix(out, "out")
    if isinstance(workspace, str):
        with _memory_of(stream):
            workspace = worker_workspace(code, A, X)
    surv = np.zeros(code.k, dtype=np.int32)
    timeline = np.zeros((code.n, 3), dtype=np.float64)
    lat = ctypes.c_double()
    _check(lib().coded_straggler_matmul(code.handle, _dtype_code(A), _ptr(A), q, r, lda, _ptr(parity), _ptr(X), s,
                                        ldx, seed, draw, shift, rate, time_unit_us, int(bool(launch_all)), _ptr(Y),
                                        _dtype_code(Y), _ptr(workspace), _ptr(out), ldo, _ptr(info),
                                        surv.ctypes.data,
                                        timeline.ctypes.data, ctypes.addressof(lat),
                                        _stream(stream)))
    return surv, timeline, lat.value


def coded_transpose(A, AT, stream=None) -> None:
    q, r, lda = _matrix(A, "A")
    r2, q2, ldat = _matrix(AT, "AT")
    if (r2, q2) != (r, q):
        raise ValueError("AT must be r x q")
    _check(lib().coded_transpose(_ptr(A), q, r, lda, _ptr(AT), ldat, _stream(stream)))


def coded_gd_sizes(codeA: Code, codeAT: Code, q: int, r: int) -> int:
    wb = ctypes.c_int64()
    _check(lib().coded_gd_sizes(codeA.handle, codeAT.handle, q, r, ctypes.addressof(wb)))
    return wb.value


def coded_gd_step(codeA: Code, codeAT: Code, A, parityA, AT, parityAT, y, x, eta: float, seed: int, iteration: int,
                  workspace, info, shift: float = 1.0, rate: float = 1.0, stream=None):
    """One coded gradient-descent iteration (x updated in place); returns both survivor sets."""
    q, r, lda = _matrix(A, "A")
    _, _, ldat = _matrix(AT, "AT")
    surv = np.zeros(codeA.k + codeAT.k, dtype=np.int32)
    _check(lib().coded_gd_step(codeA.handle, codeAT.handle, _ptr(A), lda, _ptr(parityA), _ptr(AT), ldat,
                               _ptr(parityAT), q, r, _ptr(y), _ptr(x), eta, seed, iteration, shift, rate,
                               _ptr(workspace), _ptr(info), surv.ctypes.data, _stream(stream)))
    return surv[:codeA.k], surv[codeA.k:]


def coded_simulate_runtimes(n: int, k: int, seed: int, first_draw: int, t_uncoded=None, t_repetition=None,
                            t_mds=None, shift: float = 1.0, rate: float = 1.0, stream=None) -> None:
    """Fill the given device fp64 tensors (equal lengths) with per-draw overall runtimes."""
    outs = [t for t in (t_uncoded, t_repetition, t_mds) if t is not None]
    if not outs:
        return
    count = outs[0].numel()
    if any(t.numel() != count for t in outs):
        raise ValueError("output tensors must have equal lengths")
    _check(lib().coded_simulate_runtimes(n, k, seed, first_draw, count, shift, rate, _ptr(t_uncoded),
                                         _ptr(t_repetition), _ptr(t_mds), _stream(stream)))


# ---------------------------------------------------------------- buffer helpers

def alloc_parity(code: Code, q: int, r: int, dtype, device="cuda"):
    """Parity planes of a q x r input: (planes, n-k, qb, r) of `dtype`; for a
    CODED_PLANES_LO_BF16 code (fp32 only) a flat uint8 buffer holding the fp32
    hi plane followed by the bfloat16 lo plane (see parity_planes)."""
    torch = _torch()
    qb = code.qb(q)
    if code.planes == CODED_PLANES_LO_BF16:
        if dtype != torch.float32:
            raise ValueError("a bfloat16 lo plane is for fp32 inputs")
        return torch.empty(6 * (code.n - code.k) * qb * r, dtype=torch.uint8, device=device)
    return torch.empty((code.planes, code.n - code.k, qb, r), dtype=dtype, device=device)


def parity_planes(code: Code, par, q: int, r: int):
    """(hi, lo) views of a CODED_PLANES_LO_BF16 parity buffer: hi float32 and
    lo bfloat16, each (n-k, qb, r)."""
    torch = _torch()
    shape = (code.n - code.k, code.qb(q), r)
    hb = 4 * shape[0] * shape[1] * shape[2]
    hi = par[:hb].view(torch.float32).view(shape)
    lo = par[hb:].view(torch.bfloat16).view(shape)
    return hi, lo


def alloc_y(code: Code, q: int, s: int, dtype, device="cuda"):
    torch = _torch()
    return torch.empty((code.n, code.qb(q), s), dtype=dtype, device=device)


class Shuffle:
    """Coded-shuffling master state (coded_shuffle_create): n workers, q rows, caches of cache_rows rows."""

    def __init__(self, n: int, q: int, cache_rows: int, seed: int):
        h = ctypes.c_void_p()
        _check(lib().coded_shuffle_create(n, q, cache_rows, seed, ctypes.byref(h)))
        self.handle = h
        self.n, self.q, self.cache_rows, self.seed = n, q, cache_rows, seed

    def state(self):
        """(t, partition int32[q], cache signatures uint64[q])."""
        t = ctypes.c_int64()
        assign = np.zeros(self.q, dtype=np.int32)
        sig = np.zeros(self.q, dtype=np.uint64)
        _check(lib().coded_shuffle_state(self.handle, ctypes.byref(t), assign.ctypes.data,
                                         sig.ctypes.data))
        return t.value, assign, sig

    def plan(self):
        """Plans iteration t+1: (coded_rows, terms)."""
        m, t = ctypes.c_int64(), ctypes.c_int64()
        _check(lib().coded_shuffle_plan(self.handle, ctypes.byref(m), ctypes.byref(t)))
        self.coded_rows, self.terms = m.value, t.value
        return m.value, t.value

    def tables(self):
        """The pending plan: dict of enc_off, enc_rows, term_worker, term_msg, next_assign (host arrays)."""
        out = {"enc_off": np.zeros(self.coded_rows + 1, dtype=np.int64),
               "enc_rows": np.zeros(self.terms, dtype=np.int32),
               "term_worker": np.zeros(self.terms, dtype=np.int32),
               "term_msg": np.zeros(self.terms, dtype=np.int32),
               "next_assign": np.zeros(self.q, dtype=np.int32)}
        _check(lib().coded_shuffle_tables(self.handle, *(out[k].ctypes.data for k in
                                                         ("enc_off", "enc_rows", "term_worker", "term_msg",
                                                          "next_assign"))))
        return out

    def commit(self):
        _check(lib().coded_shuffle_commit(self.handle))

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            lib().coded_shuffle_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def coded_shuffle_encode(A, enc_off, enc_rows, M, stream=None) -> None:
    """M (coded_rows x r) from A (q x r fp32) and device copies of the plan's tables."""
    q, r, lda = _matrix(A, "A")
    coded_rows, _, ldm = _matrix(M, "M")
    _check(lib().coded_shuffle_encode(_ptr(A), q, r, lda, _ptr(enc_off), _ptr(enc_rows), coded_rows,
                                      enc_rows.numel(), _ptr(M), ldm, _stream(stream)))


def coded_shuffle_decode(A, M, enc_off, enc_rows, term_msg, out, stream=None) -> None:
    """out (terms x r): each worker's decoded copy of the rows it lacked."""
    q, r, lda = _matrix(A, "A")
    coded_rows, _, ldm = _matrix(M, "M")
    _, _, ldo = _matrix(out, "out")
    _check(lib().coded_shuffle_decode(_ptr(A), q, r, lda, _ptr(M), ldm, _ptr(enc_off), _ptr(enc_rows), _ptr(term_msg),
                                      coded_rows, enc_rows.numel(), _ptr(out), ldo, _stream(stream)))



# ---------------------------------------------------------------- microscaled matrices

class MXMatrix:
    """A microscaled matrix of `cols` columns: codes (uint8, rows x code pitch) and scales (uint8,
    rows x scale pitch) in the layout of include/coded.h.  rows(a, b) is a run of its rows."""

    __slots__ = ("codes", "scales", "rows_", "cols", "fmt", "ldc", "lds")

    def __init__(self, codes, scales, cols: int, fmt: int):
        if fmt == CODED_MX4:
            need_c = (cols + 31) // 32 * 16
        elif fmt == CODED_MX8:
            need_c = (cols + 31) // 32 * 32
        else:
            raise ValueError("the format must be CODED_MX4 or CODED_MX8")
        need_s = (cols + 127) // 128 * 4
        uint8 = _torch().uint8
        if codes.dtype is not uint8 or scales.dtype is not uint8 or codes.dim() != 2 or scales.dim() != 2:
            raise ValueError("codes and scales must be uint8, rows of bytes")
        n, width = codes.shape
        n_s, width_s = scales.shape
        ldc, step = codes.stride()
        lds, step_s = scales.stride()
        if width < need_c or (need_c and step != 1):
            raise ValueError(f"codes must be rows of at least {need_c} bytes")
        if width_s < need_s or (need_s and step_s != 1):
            raise ValueError(f"scales must be rows of at least {need_s} bytes")
        if n != n_s:
            raise ValueError("codes and scales must have the same number of rows")
        self.codes, self.scales, self.rows_, self.cols, self.fmt = codes, scales, n, cols, fmt
        self.ldc, self.lds = (ldc, lds) if n > 1 and cols > 0 else (need_c, need_s)

    @property
    def shape(self):
        return self.rows_, self.cols

    def rows(self, begin: int, end: int) -> "MXMatrix":
        return MXMatrix(self.codes[begin:end], self.scales[begin:end], self.cols, self.fmt)

    def _args(self):
        return self.fmt, self.codes.data_ptr(), self.ldc, self.scales.data_ptr(), self.lds


def _mx_dense(t, name):
    """(rows, cols, row stride, type) of a 1-D (column) or row-major 2-D tensor; the stride of a
    dimension of size 1 is not looked at."""
    try:
        dt = _dtype_code(t)
    except KeyError:
        raise ValueError(f"{name} must be float32 or bfloat16") from None
    if t.dim() == 1:
        rows, cols, ld, step = t.shape[0], 1, t.stride(0), 1
    elif t.dim() == 2:
        rows, cols = t.shape
        ld, step = t.stride()
    else:
        raise ValueError(f"{name} must be 1-D or 2-D")
    if cols > 1 and step != 1 and rows > 0:
        raise ValueError(f"{name} must be row-major")
    return rows, cols, ld if rows > 1 else max(cols, 1), dt


@functools.lru_cache(maxsize=256)
def coded_mx_sizes(fmt: int, r: int):
    """(code pitch, scale pitch) in bytes of rows of r columns."""
    c, s = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().coded_mx_sizes(fmt, r, ctypes.addressof(c), ctypes.addressof(s)))
    return c.value, s.value


def alloc_mx(q: int, r: int, fmt: int, device="cuda") -> MXMatrix:
    """Room for a q x r microscaled matrix (not cleared: coded_mx_quantize writes all that is read)."""
    torch = _torch()
    c, s = coded_mx_sizes(fmt, r)
    empty, uint8 = torch.empty, torch.uint8
    return MXMatrix(empty((q, c), dtype=uint8, device=device), empty((q, s), dtype=uint8, device=device), r, fmt)


def coded_mx_quantize(A, M: MXMatrix, stream=None) -> None:
    """Codes and scales of A (float32 or bfloat16) into M."""
    q, r, lda, dt = _mx_dense(A, "A")
    if M.shape != (q, r):
        raise ValueError("M must have A's shape")
    _check(lib().coded_mx_quantize(dt, A.data_ptr(), q, r, lda, *M._args(), _stream(stream)))


def coded_mx_dequantize(M: MXMatrix, out, stream=None) -> None:
    """M's values into out (float32 or bfloat16)."""
    q, r, ldo, dt = _mx_dense(out, "out")
    if M.shape != (q, r):
        raise ValueError("out must have M's shape")
    _check(lib().coded_mx_dequantize(*M._args(), q, r, dt, out.data_ptr(), ldo, _stream(stream)))


@functools.lru_cache(maxsize=256)
def coded_mx_workspace(transposed: bool, fmt: int, q: int, r: int, x_dt: int, s: int, x_rows: bool = False,
                       y_rows: bool = False) -> int:
    """Bytes of workspace of coded_mx_mm, or of coded_mx_mm_t when transposed."""
    b = ctypes.c_int64()
    _check(lib().coded_mx_workspace(int(bool(transposed)), fmt, q, r, x_dt, s, bool(x_rows) | bool(y_rows) << 1,
                                    ctypes.addressof(b)))
    return b.value


def _mx_side(t, name, by_rows):
    """(terms, right-hand sides, row stride, type) of X or Y; a 1-D tensor is one right-hand side."""
    rows, cols, ld, dt = _mx_dense(t, name)
    if not by_rows:
        return rows, cols, ld, dt
    if t.dim() == 1:
        if rows > 1 and ld != 1:
            raise ValueError(f"{name} must be contiguous")
        return rows, 1, max(rows, 1), dt
    return cols, rows, ld, dt


def _mx_product(transposed, M, X, Y, x_rows, y_rows, alpha, beta, C, workspace, stream):
    q, r = M.shape
    k, n = (q, r) if transposed else (r, q)
    if isinstance(X, MXMatrix):
        if not x_rows:
            raise ValueError("a microscaled X holds a right-hand side a row: x_rows=True")
        x_dt, xp, ldx, xsp, ldxs = X._args()
        s, kx = X.shape
    else:
        kx, s, ldx, x_dt = _mx_side(X, "X", x_rows)
        xp, xsp, ldxs = X.data_ptr(), None, 0
    if kx != k:
        raise ValueError(f"X must have {k} terms a right-hand side")
    ny, sy, ldy, y_dt = _mx_side(Y, "Y", y_rows)
    if ny != n or sy != s:
        raise ValueError(f"Y must have {n} results for each of {s} right-hand sides")
    cp, ldcc = None, 0
    if beta != 0:
        if C is None or C.dtype != Y.dtype:
            raise ValueError("C must be given, of Y's type, when beta is not 0")
        if C.shape == Y.shape:
            ldcc = _mx_side(C, "C", y_rows)[2]
        elif C.dim() == 1 and Y.dim() == 2 and C.shape[0] == Y.shape[1] and (C.shape[0] < 2 or C.stride(0) == 1):
            ldcc = 0   # one row for every row of Y
        else:
            raise ValueError("C must have Y's shape, or be one row of it")
        cp = C.data_ptr()
    wsp, wsb = None, 0
    if isinstance(workspace, str):
        wsb = coded_mx_workspace(transposed, M.fmt, q, r, x_dt, s, x_rows, y_rows)
        if wsb:
            torch = _torch()
            if stream is None:   # the usual call: 0.4 us less than by way of a context
                workspace = torch.empty(wsb, dtype=torch.uint8, device=Y.device)
            else:
                with _memory_of(stream):
                    workspace = torch.empty(wsb, dtype=torch.uint8, device=Y.device)
            wsp = workspace.data_ptr()
    elif workspace is not None:
        wsp, wsb = _given(workspace)
    order = bool(x_rows) | bool(y_rows) << 1
    if transposed:
        _check(lib().coded_mx_mm_t(*M._args(), q, r, x_dt, xp, ldx, s, order, alpha, beta, cp, ldcc, Y.data_ptr(), y_dt,
                                   ldy, wsp, wsb, _stream(stream)))
    else:
        _check(lib().coded_mx_mm(*M._args(), q, r, x_dt, xp, ldx, xsp, ldxs, s, order, alpha, beta, cp, ldcc,
                                 Y.data_ptr(), y_dt, ldy, wsp, wsb, _stream(stream)))


def coded_mx_mm(M: MXMatrix, X, Y, x_rows: bool = False, y_rows: bool = False, alpha: float = 1.0, beta: float = 0.0,
                C=None, workspace="auto", stream=None) -> None:
    """Y = alpha * M X + beta * C.  X: r x s (or s x r with x_rows; then an MXMatrix too); Y: q x s (or s x q with
    y_rows); C: like Y, or one row of it for every row.  A 1-D X, Y is one right-hand side.
    workspace: "auto", or a device buffer of coded_mx_workspace bytes."""
    _mx_product(False, M, X, Y, x_rows, y_rows, alpha, beta, C, workspace, stream)


def coded_mx_mm_t(M: MXMatrix, U, Z, x_rows: bool = False, y_rows: bool = False, alpha: float = 1.0, beta: float = 0.0,
                  C=None, workspace="auto", stream=None) -> None:
    """Z = alpha * M^T U + beta * C.  U: q x s (or s x q with x_rows); Z: r x s (or s x r with y_rows)."""
    if isinstance(U, MXMatrix):
        raise ValueError("U must be float32 or bfloat16")
    _mx_product(True, M, U, Z, x_rows, y_rows, alpha, beta, C, workspace, stream)


# ---------------------------------------------------------------- matrices in 8 bits, dropout, embeddings

def _on_gpu(names, tensors):
    """Every tensor (None: left out) must be in the current device's memory: another device's, or the host's, would fault."""
    device = -2
    for name, t in zip(names, tensors):
        if t is None:
            continue
        at = t.get_device()      # -1: the host
        if at < 0:
            raise ValueError(f"{name} must be on the GPU")
        if device == -2:
            device = _torch().cuda.current_device()
        if at != device:
            raise ValueError(f"{name} must be on the current device, {device}")


def _workspace(nbytes, device, stream):
    torch = _torch()
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with _memory_of(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


class F8Matrix:
    """A rows x cols matrix in 8 bits: codes (uint8, rows x code pitch) and scales (float32, a row for every 128
    columns, an element for every block_rows rows) in the layout of include/coded.h.  block_rows: 1 or 128."""

    __slots__ = ("codes", "scales", "rows_", "cols", "block_rows", "ldc", "lds")

    def __init__(self, codes, scales, rows: int, cols: int, block_rows: int = 1):
        torch = _torch()
        if block_rows not in (1, 128):
            raise ValueError("a block must have 1 or 128 rows")
        blocks, groups = (cols + 127) // 128, (rows + block_rows - 1) // block_rows
        width = blocks * 128
        if codes.dtype is not torch.uint8 or scales.dtype is not torch.float32 or codes.dim() != 2 or scales.dim() != 2:
            raise ValueError("codes must be uint8 and scales float32, both 2-D")
        n, wide = codes.shape
        n_s, wide_s = scales.shape
        ldc, step = codes.stride()
        lds, step_s = scales.stride()
        if rows < 0 or cols < 0 or n != rows or wide < width or (width and step != 1):
            raise ValueError(f"codes must be {rows} rows of at least {width} bytes")
        if n_s < blocks or wide_s < groups or (groups > 1 and step_s != 1):
            raise ValueError(f"scales must be {blocks} rows of at least {groups} elements")
        self.codes, self.scales, self.rows_, self.cols, self.block_rows = codes, scales, rows, cols, block_rows
        self.ldc = ldc if rows > 1 and cols > 0 else width
        self.lds = lds if blocks > 1 else groups

    @property
    def shape(self):
        return self.rows_, self.cols

    def rows(self, begin: int, end: int) -> "F8Matrix":
        """Rows begin .. end - 1; begin must be a multiple of block_rows."""
        if not 0 <= begin <= end <= self.rows_ or begin % self.block_rows:
            raise ValueError("a run of rows must lie within the matrix and begin with a block")
        at = begin // self.block_rows
        return F8Matrix(self.codes[begin:end], self.scales[:, at:], end - begin, self.cols, self.block_rows)

    def _args(self):
        return self.block_rows, self.codes.data_ptr(), self.ldc, self.scales.data_ptr(), self.lds


def coded_f8_sizes(q: int, r: int, block_rows: int = 1):
    """(code pitch in bytes, scale pitch in elements) of a q x r matrix."""
    c, s = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().coded_f8_sizes(q, r, block_rows, ctypes.addressof(c), ctypes.addressof(s)))
    return c.value, s.value


def alloc_f8(q: int, r: int, block_rows: int = 1, device="cuda") -> F8Matrix:
    """Room for a q x r matrix in 8 bits (not cleared: coded_f8_quantize writes all that is read)."""
    torch = _torch()
    if q < 0 or r < 0 or block_rows not in (1, 128):
        raise ValueError("sizes must be >= 0 and a block have 1 or 128 rows")
    blocks = (r + 127) // 128
    width, groups = blocks * 128, (q + block_rows - 1) // block_rows
    M = F8Matrix.__new__(F8Matrix)      # what its checks would find is known
    M.codes = torch.empty((q, width), dtype=torch.uint8, device=device)
    M.scales = torch.empty((blocks, groups), dtype=torch.float32, device=device)
    M.rows_, M.cols, M.block_rows, M.ldc, M.lds = q, r, block_rows, width, groups
    return M


def coded_f8_quantize(A, M: "F8Matrix | None" = None, MT: "F8Matrix | None" = None, stream=None) -> None:
    """Codes and scales of A (float32 or bfloat16) into M, of its transpose into MT, or both in one pass."""
    q, r, lda, dt = _mx_dense(A, "A")
    if M is None and MT is None:
        raise ValueError("M or MT must be given")
    if M is not None and M.shape != (q, r):
        raise ValueError("M must have A's shape")
    if MT is not None and MT.shape != (r, q):
        raise ValueError("MT must have the shape of A's transpose")
    _on_gpu(("A", "M", "M", "MT", "MT"), (A, *((None, None) if M is None else (M.codes, M.scales)),
                                          *((None, None) if MT is None else (MT.codes, MT.scales))))
    none = 1, None, 0, None, 0
    _check(lib().coded_f8_quantize(dt, A.data_ptr(), q, r, lda, *(none if M is None else M._args()),
                                   *(none if MT is None else MT._args()), _stream(stream)))


def coded_f8_dequantize(M: F8Matrix, out, stream=None) -> None:
    """M's values into out (float32 or bfloat16)."""
    q, r, ldo, dt = _mx_dense(out, "out")
    if M.shape != (q, r):
        raise ValueError("out must have M's shape")
    _on_gpu(("out", "M", "M"), (out, M.codes, M.scales))
    _check(lib().coded_f8_dequantize(q, r, *M._args(), dt, out.data_ptr(), ldo, _stream(stream)))


@functools.lru_cache(maxsize=256)
def coded_f8_workspace(q: int, r: int, s: int, y_dt: int, y_rows: bool = False) -> int:
    """Bytes of workspace of coded_f8_mm."""
    b = ctypes.c_int64()
    _check(lib().coded_f8_workspace(q, r, s, y_dt, bool(y_rows) << 1, ctypes.addressof(b)))
    return b.value


def coded_f8_mm(A: F8Matrix, X: F8Matrix, Y, y_rows: bool = False, alpha: float = 1.0, beta: float = 0.0, C=None,
                workspace="auto", stream=None) -> None:
    """Y = alpha * A X^T + beta * C.  A: q x r, X: s x r; Y: q x s (or s x q with y_rows); C: like Y, or one row of it
    for every row.  A 1-D Y is one right-hand side.  workspace: "auto", or a device buffer of coded_f8_workspace bytes."""
    q, r = A.shape
    s, rx = X.shape
    if rx != r:
        raise ValueError(f"X must have {r} columns")
    ny, sy, ldy, y_dt = _mx_side(Y, "Y", y_rows)
    if ny != q or sy != s:
        raise ValueError(f"Y must have {q} results for each of {s} right-hand sides")
    cp, ldcc = None, 0
    if beta != 0:
        if C is None or C.dtype != Y.dtype:
            raise ValueError("C must be given, of Y's type, when beta is not 0")
        if C.shape == Y.shape:
            ldcc = _mx_side(C, "C", y_rows)[2]
        elif C.dim() == 1 and Y.dim() == 2 and C.shape[0] == Y.shape[1] and (C.shape[0] < 2 or C.stride(0) == 1):
            ldcc = 0   # one row for every row of Y
        else:
            raise ValueError("C must have Y's shape, or be one row of it")
        cp = C.data_ptr()
    wsp, wsb = None, 0
    if not (workspace is None or isinstance(workspace, str)):
        wsp, wsb = _given(workspace)
    _on_gpu(("Y", "A", "A", "X", "X", "C", "workspace"), (Y, A.codes, A.scales, X.codes, X.scales, C if beta != 0 else None,
                                                        None if isinstance(workspace, str) else workspace))
    if isinstance(workspace, str):
        wsb = coded_f8_workspace(q, r, s, y_dt, y_rows)
        if wsb:
            workspace = _workspace(wsb, Y.device, stream)
            wsp = workspace.data_ptr()
    _check(lib().coded_f8_mm(q, r, s, *A._args(), *X._args(), bool(y_rows) << 1, alpha, beta, cp, ldcc, Y.data_ptr(), y_dt, ldy,
                             wsp, wsb, _stream(stream)))


def coded_dropout(X, out, p: float, seed: int, draw: int, first_row: int = 0, C=None, stream=None) -> None:
    """out = X / (1 - p) where an element is kept and 0 where it is dropped, plus C.  The mask is a function of seed,
    draw and an element's place; X holds rows first_row .. of the whole batch.  out may be X or C."""
    q, r, ldx, dt = _mx_dense(X, "X")
    qo, ro, ldo, dto = _mx_dense(out, "out")
    if (qo, ro) != (q, r) or dto != dt:
        raise ValueError("out must have X's shape and type")
    ldcc = 0
    if C is not None:
        qc, rc, ldcc, dtc = _mx_dense(C, "C")
        if (qc, rc) != (q, r) or dtc != dt:
            raise ValueError("C must have X's shape and type")
    if not 0 <= seed < 1 << 64 or not 0 <= draw < 1 << 56:
        raise ValueError("seed must be in [0, 2^64) and draw in [0, 2^56)")
    _on_gpu(("X", "out", "C"), (X, out, C))
    _check(lib().coded_dropout(dt, X.data_ptr(), q, r, ldx, p, seed, draw, first_row, _ptr(C), ldcc, out.data_ptr(), ldo,
                               _stream(stream)))


def _tokens(tok):
    """(data, bytes a token, tokens) of a contiguous int32 or int64 tensor of any shape."""
    torch = _torch()
    if tok.dtype not in (torch.int32, torch.int64) or not tok.is_contiguous():
        raise ValueError("tokens must be int32 or int64, contiguous")
    return tok.data_ptr(), tok.element_size(), tok.numel()


def coded_embed(E, tok, out, scale: float = 1.0, skip: int = -1, stream=None) -> None:
    """out[i] = scale * E[tok[i]] (E: vocab x d, out: n x d); zero for the token `skip`, NaN for one that E lacks
    (-1 too: a skip that is no row of E skips none)."""
    vocab, d, lde, e_dt = _mx_dense(E, "E")
    n_out, d_out, ldo, out_dt = _mx_dense(out, "out")
    tp, size, n = _tokens(tok)
    if E.dim() != 2 or out.dim() != 2 or (n_out, d_out) != (n, d):
        raise ValueError(f"out must be {n} rows of {d}")
    _on_gpu(("E", "tok", "out"), (E, tok, out))
    _check(lib().coded_embed(e_dt, E.data_ptr(), vocab, d, lde, tp, size, n, skip, scale, out_dt, out.data_ptr(), ldo, _stream(stream)))


@functools.lru_cache(maxsize=256)
def coded_embed_workspace(n: int, vocab: int, d: int) -> int:
    """Bytes of workspace of coded_embed_grad."""
    b = ctypes.c_int64()
    _check(lib().coded_embed_workspace(n, vocab, d, ctypes.addressof(b)))
    return b.value


def coded_embed_grad(G, tok, dE, scale: float = 1.0, beta: float = 0.0, skip: int = -1, workspace="auto", stream=None) -> None:
    """dE[v] = beta * dE[v] + scale * the sum of the rows G[i] with tok[i] == v (G: n x d, dE: vocab x d).
    workspace: "auto", or a device buffer of coded_embed_workspace bytes."""
    n_g, d_g, ldg, g_dt = _mx_dense(G, "G")
    vocab, d, ldde, e_dt = _mx_dense(dE, "dE")
    tp, size, n = _tokens(tok)
    if G.dim() != 2 or dE.dim() != 2 or (n_g, d_g) != (n, d):
        raise ValueError(f"G must be {n} rows of {d}")
    wsp, wsb = None, 0
    if not (workspace is None or isinstance(workspace, str)):
        wsp, wsb = _given(workspace)
    _on_gpu(("G", "tok", "dE", "workspace"), (G, tok, dE, None if isinstance(workspace, str) else workspace))
    if isinstance(workspace, str):
        wsb = coded_embed_workspace(n, vocab, d)
        if wsb:
            workspace = _workspace(wsb, dE.device, stream)
            wsp = workspace.data_ptr()
    _check(lib().coded_embed_grad(g_dt, G.data_ptr(), n, d, ldg, tp, size, vocab, skip, scale, beta, e_dt, dE.data_ptr(), ldde, wsp,
                                  wsb, _stream(stream)))
