"""ctypes binding of include/pf_layer.h: the operators of a layer around the delta rule.  Argument marshalling only, as in
binding.py: every step of the computation runs in the HIP kernels of libpf_layer.so, PyTorch supplies device memory and the
stream, and without the library this module raises.

The functions without the pf_ prefix take torch tensors on the GPU, check them, allocate the outputs (and a workspace unless
one is handed in) and make one library call on the current stream of the tensors' device, or on `stream`.
"""
from __future__ import annotations

import ctypes
import os

from .binding import PF_BF16, PF_F32, PF_OK, PfError, _ptr, _stream_handle

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libpf_layer.so")

PF_GATE_VALUE, PF_GATE_LOG, PF_GATE_LOGIT = range(3)
GATES = {"value": PF_GATE_VALUE, "log": PF_GATE_LOG, "logit": PF_GATE_LOGIT}

EXPORTS = ["pf_norm_supported", "pf_norm_fwd", "pf_norm_bwd_workspace_bytes", "pf_norm_bwd", "pf_quant_fp8",
           "pf_matmul_fp8_workspace_bytes", "pf_matmul_fp8", "pf_gated_workspace_bytes", "pf_gated_fwd", "pf_gated_bwd"]


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2504_00492_amd.build` "
                          "(there is no fallback path)")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i, ll, sz, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t, ctypes.c_float
    for name, res, args in (
            ("pf_norm_supported", i, [i, i]),
            ("pf_norm_fwd", i, [vp, ll, vp, ll, vp, vp, vp, vp, ll, vp, i, i, f, i, vp]),
            ("pf_norm_bwd_workspace_bytes", sz, [i, i]),
            ("pf_norm_bwd", i, [vp, ll, vp, vp, ll, vp, ll, vp, vp, i, i, f, i, vp, sz, vp]),
            ("pf_quant_fp8", i, [vp, ll, vp, ll, vp, vp, ll, vp, i, i, i, i, vp]),
            ("pf_matmul_fp8_workspace_bytes", sz, [i, i, i, i]),
            ("pf_matmul_fp8", i, [vp, ll, vp, vp, ll, vp, i, vp, ll, i, i, i, i, vp, sz, vp]),
            ("pf_gated_workspace_bytes", sz, [i, i, i, i]),
            ("pf_gated_fwd", i, [vp, ll, ll, vp, ll, ll, vp, vp, vp, i, i, i, i, i, i, vp, sz, vp]),
            ("pf_gated_bwd", i, [vp, ll, ll, vp, ll, ll, vp, vp, vp, ll, ll, vp, vp, vp, vp, i, i, i, i, i, i, vp, sz, vp])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


_lib = _load()


# ---- the library's calls, raw: pointers may be torch tensors, ints or None; they return the pf_status

def pf_norm_supported(D, dt) -> int:
    return int(_lib.pf_norm_supported(D, dt))


def pf_norm_fwd(X, ldx, R, ldr, w, S, Y, Q, ldq, scale, M, D, eps, dt, stream=None) -> int:
    return int(_lib.pf_norm_fwd(_ptr(X), ldx, _ptr(R), ldr, _ptr(w), _ptr(S), _ptr(Y), _ptr(Q), ldq, _ptr(scale), M, D, eps, dt,
                                _stream_handle(stream)))


def pf_norm_bwd_workspace_bytes(M, D) -> int:
    return int(_lib.pf_norm_bwd_workspace_bytes(M, D))


def pf_norm_bwd(S, lds, w, dY, lddy, dS, ldds, dX, dw, M, D, eps, dt, workspace, workspace_bytes, stream=None) -> int:
    return int(_lib.pf_norm_bwd(_ptr(S), lds, _ptr(w), _ptr(dY), lddy, _ptr(dS), ldds, _ptr(dX), _ptr(dw), M, D, eps, dt,
                                _ptr(workspace), workspace_bytes, _stream_handle(stream)))


def pf_quant_fp8(X, ldx, Q, ldq, scale, QT, ldqt, scaleT, M, K, rows, dt, stream=None) -> int:
    return int(_lib.pf_quant_fp8(_ptr(X), ldx, _ptr(Q), ldq, _ptr(scale), _ptr(QT), ldqt, _ptr(scaleT), M, K, rows, dt,
                                 _stream_handle(stream)))


def pf_matmul_fp8_workspace_bytes(M, N, K, b_rows) -> int:
    return int(_lib.pf_matmul_fp8_workspace_bytes(M, N, K, b_rows))


def pf_matmul_fp8(A, lda, sa, B, ldb, sb, b_rows, C, ldc, M, N, K, dt, workspace, workspace_bytes, stream=None) -> int:
    return int(_lib.pf_matmul_fp8(_ptr(A), lda, _ptr(sa), _ptr(B), ldb, _ptr(sb), b_rows, _ptr(C), ldc, M, N, K, dt,
                                  _ptr(workspace), workspace_bytes, _stream_handle(stream)))


def pf_gated_workspace_bytes(B, L, D, dt) -> int:
    return int(_lib.pf_gated_workspace_bytes(B, L, D, dt))


def pf_gated_fwd(X, xb, xt, G, gb, gt, h0, Y, hL, B, L, D, gate, mix, dt, workspace, workspace_bytes, stream=None) -> int:
    return int(_lib.pf_gated_fwd(_ptr(X), xb, xt, _ptr(G), gb, gt, _ptr(h0), _ptr(Y), _ptr(hL), B, L, D, gate, mix, dt,
                                 _ptr(workspace), workspace_bytes, _stream_handle(stream)))


def pf_gated_bwd(X, xb, xt, G, gb, gt, h0, Y, dY, dyb, dyt, dhL, dX, dG, dh0, B, L, D, gate, mix, dt, workspace,
                 workspace_bytes, stream=None) -> int:
    return int(_lib.pf_gated_bwd(_ptr(X), xb, xt, _ptr(G), gb, gt, _ptr(h0), _ptr(Y), _ptr(dY), dyb, dyt, _ptr(dhL), _ptr(dX),
                                 _ptr(dG), _ptr(dh0), B, L, D, gate, mix, dt, _ptr(workspace), workspace_bytes,
                                 _stream_handle(stream)))


# ---- on torch tensors

def _dt(t, what):
    import torch
    if t.dtype == torch.bfloat16:
        return PF_BF16
    if t.dtype == torch.float32:
        return PF_F32
    raise ValueError(f"{what} must be float32 or bfloat16")


def _check(t, what, shape, dtype, device, dense=True):
    """t: None, or a tensor of this shape, type and device whose innermost dimension is contiguous (dense: all of it)."""
    if t is None:
        return
    if t.device != device:
        raise ValueError(f"{what} must be on {device}; there is no CPU path")
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    if dense and not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if not dense and t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the innermost dimension of {what} must be contiguous")


def _gpu(t, what):
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA (HIP) tensor; there is no CPU path")
    return t.device


def _row(t):
    """Row stride of a matrix (any value serves where there is but one row)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))


def _byte_rows(M, K, device):
    """An uninitialised e4m3 matrix whose rows lie a multiple of 16 bytes apart."""
    import torch
    ld = (K + 15) // 16 * 16
    q = torch.empty((M, ld), dtype=torch.float8_e4m3fn, device=device)
    return q if ld == K else q[:, :K]


def _byte_row(t, what):
    """Row stride of an e4m3 matrix, whose last row too must be held in whole 16 bytes."""
    rows, whole = t.shape[0], (t.shape[1] + 15) // 16 * 16
    ld = t.stride(0) if rows > 1 else max(whole, t.stride(0) // 16 * 16)
    if rows and t.storage_offset() + (rows - 1) * ld + whole > t.untyped_storage().nbytes():
        raise ValueError(f"the rows of {what} must be held in a multiple of 16 bytes")
    return ld


def _stream_of(device, stream):
    import torch
    return torch._C._cuda_getCurrentRawStream(device.index) if stream is None else _stream_handle(stream)


def _call(fn, name, device, args):
    """One library call with `device` as the current one."""
    import torch
    if torch._C._cuda_getDevice() == device.index:
        st = fn(*args)
    else:
        with torch.cuda.device(device):
            st = fn(*args)
    if st != PF_OK:
        raise PfError(st, name)


def _workspace(need, given, device):
    """(address, bytes) of the workspace handed in, or of a new one; the tensor is kept until the call has been made."""
    import torch
    if given is None:
        if not need:
            return None, None, 0
        given = torch.empty(need, dtype=torch.uint8, device=device)
    return given, given.data_ptr(), given.numel() * given.element_size()


def norm_fwd(X, w=None, R=None, *, eps, y: bool = True, fp8: bool = False, inplace: bool = False, stream=None):
    """Root-mean-square norm of the rows of X + R (pf_norm_fwd).  X, R [M, D] (float32 or bfloat16, rows may lie apart), w [D]
    of the same type.  Returns (S, Y, Q, scale): S the stored sum (X itself without R; R's own memory with inplace, which
    asks for a contiguous R), Y the norm (None with y=False), Q and scale the norm in 8 bits (None unless fp8)."""
    import torch
    device, dt = _gpu(X, "X"), _dt(X, "X")
    if X.dim() != 2:
        raise ValueError("X must have two dimensions")
    M, D = X.shape
    _check(X, "X", (M, D), X.dtype, device, dense=False)
    _check(R, "R", (M, D), X.dtype, device, dense=inplace)
    _check(w, "w", (D,), X.dtype, device)
    if not (y or fp8):
        raise ValueError("neither y nor fp8 is wanted")
    if inplace and R is None:
        raise ValueError("inplace needs R")
    S = X if R is None else R if inplace else torch.empty((M, D), dtype=X.dtype, device=device)
    Y = torch.empty((M, D), dtype=X.dtype, device=device) if y else None
    Q = scale = None
    if fp8:
        Q, scale = _byte_rows(M, D, device), torch.empty((-(-D // 128), M), dtype=torch.float32, device=device)
    _call(_lib.pf_norm_fwd, "pf_norm_fwd", device, (
        X.data_ptr(), _row(X), _ptr(R), 0 if R is None else _row(R), _ptr(w), None if R is None else S.data_ptr(), _ptr(Y), _ptr(Q),
        (D + 15) // 16 * 16, _ptr(scale), M, D, eps, dt, _stream_of(device, stream)))
    return S, Y, Q, scale


def norm_bwd(S, dY, w=None, dS=None, *, eps, want_dw: bool = True, workspace=None, stream=None):
    """Backward of norm_fwd (pf_norm_bwd): S the stored sum, dY the gradient of the norm, dS that of the sum past the norm
    (None: none).  Returns (dX, dw): dX [M, D] in the inputs' type, dw [D] in float32 (None unless wanted)."""
    import torch
    device, dt = _gpu(S, "S"), _dt(S, "S")
    if S.dim() != 2:
        raise ValueError("S must have two dimensions")
    M, D = S.shape
    _check(S, "S", (M, D), S.dtype, device, dense=False)
    _check(dY, "dY", (M, D), S.dtype, device, dense=False)
    _check(dS, "dS", (M, D), S.dtype, device, dense=False)
    _check(w, "w", (D,), S.dtype, device)
    dX = torch.empty((M, D), dtype=S.dtype, device=device)
    dw = torch.empty(D, dtype=torch.float32, device=device) if want_dw else None
    keep, wp, wb = _workspace(_lib.pf_norm_bwd_workspace_bytes(M, D) if want_dw else 0, workspace, device)
    _call(_lib.pf_norm_bwd, "pf_norm_bwd", device, (
        S.data_ptr(), _row(S), _ptr(w), dY.data_ptr(), _row(dY), _ptr(dS), 0 if dS is None else _row(dS), dX.data_ptr(), _ptr(dw),
        M, D, eps, dt, wp, wb, _stream_of(device, stream)))
    return dX, dw


def quant_fp8(X, *, rows: int = 1, plain: bool = True, transposed: bool = False, stream=None):
    """X [M, K] (float32 or bfloat16, rows may lie apart) in 8 bits (pf_quant_fp8), with a scale for each row and 128 columns
    (rows=1) or each 128 x 128 (rows=128).  Returns (Q, scale, QT, scaleT); Q and scale are None with plain=False, QT and
    scaleT (the transposed matrix, its blocks along its own rows) unless transposed."""
    import torch
    device, dt = _gpu(X, "X"), _dt(X, "X")
    if X.dim() != 2:
        raise ValueError("X must have two dimensions")
    M, K = X.shape
    _check(X, "X", (M, K), X.dtype, device, dense=False)
    if rows not in (1, 128):
        raise ValueError("rows must be 1 or 128")
    if not (plain or transposed):
        raise ValueError("neither plain nor transposed is wanted")
    Q = scale = QT = scaleT = None
    per = lambda n: n if rows == 1 else -(-n // 128)      # noqa: E731
    if plain:
        Q, scale = _byte_rows(M, K, device), torch.empty((-(-K // 128), per(M)), dtype=torch.float32, device=device)
    if transposed:
        QT, scaleT = _byte_rows(K, M, device), torch.empty((-(-M // 128), per(K)), dtype=torch.float32, device=device)
    _call(_lib.pf_quant_fp8, "pf_quant_fp8", device, (
        X.data_ptr(), _row(X), _ptr(Q), (K + 15) // 16 * 16, _ptr(scale), _ptr(QT), (M + 15) // 16 * 16, _ptr(scaleT), M, K, rows,
        dt, _stream_of(device, stream)))
    return Q, scale, QT, scaleT


def matmul_fp8(A, sa, B, sb, *, b_rows: int = 128, out_dtype=None, workspace=None, stream=None):
    """C [M, N] = A [M, K] times B [N, K] transposed, both e4m3 with scales (pf_matmul_fp8): sa [ceil(K/128), M], sb
    [ceil(K/128), N] (b_rows=1) or [ceil(K/128), ceil(N/128)] (b_rows=128).  Rows of A and B lie a multiple of 16 bytes apart,
    as quant_fp8 and norm_fwd lay them.  out_dtype: bfloat16 (the default) or float32."""
    import torch
    device = _gpu(A, "A")
    if A.dim() != 2 or B.dim() != 2:
        raise ValueError("A and B must have two dimensions")
    if b_rows not in (1, 128):
        raise ValueError("b_rows must be 1 or 128")
    out_dtype = torch.bfloat16 if out_dtype is None else out_dtype
    (M, K), N = A.shape, B.shape[0]
    nk = -(-K // 128)
    _check(A, "A", (M, K), torch.float8_e4m3fn, device, dense=False)
    _check(B, "B", (N, K), torch.float8_e4m3fn, device, dense=False)
    _check(sa, "sa", (nk, M), torch.float32, device)
    _check(sb, "sb", (nk, N if b_rows == 1 else -(-N // 128)), torch.float32, device)
    C = torch.empty((M, N), dtype=out_dtype, device=device)
    dt = _dt(C, "out_dtype")
    keep, wp, wb = _workspace(_lib.pf_matmul_fp8_workspace_bytes(M, N, K, b_rows), workspace, device)
    _call(_lib.pf_matmul_fp8, "pf_matmul_fp8", device, (
        A.data_ptr(), _byte_row(A, "A"), sa.data_ptr(), B.data_ptr(), _byte_row(B, "B"), sb.data_ptr(), b_rows, C.data_ptr(), N, M, N,
        K, dt, wp, wb, _stream_of(device, stream)))
    return C


def _gate_of(gate):
    if gate not in GATES:
        raise ValueError(f"gate must be one of {', '.join(GATES)}")
    return GATES[gate]


def _steps(t):
    """Batch and token strides of [B, L, D] (where there is but one of them, what a dense array would have)."""
    B, L, D = t.shape
    token = t.stride(1) if L > 1 else D
    return (t.stride(0) if B > 1 else L * token), token


def gated_fwd(X, G, h0=None, *, gate: str = "log", mix: bool = False, workspace=None, stream=None):
    """The gated linear recurrence h_t = a_t h_{t-1} + b_t (pf_gated_fwd): a = G, exp(G) or its sigmoid by gate ("value",
    "log", "logit"), b = X, or (1 - a) X with mix.  X, G [B, L, D] (float32 or bfloat16, tokens and sequences may lie apart or in the
    other order), h0 [B, D] float32 or None.  Returns (Y [B, L, D], h_L [B, D] float32)."""
    import torch
    device, dt, form = _gpu(X, "X"), _dt(X, "X"), _gate_of(gate)
    if X.dim() != 3:
        raise ValueError("X must have three dimensions")
    B, L, D = X.shape
    _check(X, "X", (B, L, D), X.dtype, device, dense=False)
    _check(G, "G", (B, L, D), X.dtype, device, dense=False)
    _check(h0, "h0", (B, D), torch.float32, device)
    Y = torch.empty((B, L, D), dtype=X.dtype, device=device)
    hL = torch.empty((B, D), dtype=torch.float32, device=device)
    keep, wp, wb = _workspace(_lib.pf_gated_workspace_bytes(B, L, D, dt), workspace, device)
    _call(_lib.pf_gated_fwd, "pf_gated_fwd", device, (
        X.data_ptr(), *_steps(X), G.data_ptr(), *_steps(G), _ptr(h0), Y.data_ptr(), hL.data_ptr(), B, L, D, form, int(mix), dt, wp, wb,
        _stream_of(device, stream)))
    return Y, hL


def gated_bwd(X, G, Y, dY, h0=None, dhL=None, *, gate: str = "log", mix: bool = False, workspace=None, stream=None):
    """Backward of gated_fwd (pf_gated_bwd) from what it was given and returned (X may be None without mix), dY the gradient of
    Y, dhL that of h_L (float32, None: none).  Returns (dX, dG, dh0)."""
    import torch
    device, dt, form = _gpu(G, "G"), _dt(G, "G"), _gate_of(gate)
    if G.dim() != 3:
        raise ValueError("G must have three dimensions")
    if mix and X is None:
        raise ValueError("mix needs X")
    B, L, D = G.shape
    _check(X, "X", (B, L, D), G.dtype, device, dense=False)
    _check(G, "G", (B, L, D), G.dtype, device, dense=False)
    _check(Y, "Y", (B, L, D), G.dtype, device)
    _check(dY, "dY", (B, L, D), G.dtype, device, dense=False)
    _check(h0, "h0", (B, D), torch.float32, device)
    _check(dhL, "dhL", (B, D), torch.float32, device)
    dX, dG = (torch.empty((B, L, D), dtype=G.dtype, device=device) for _ in range(2))
    dh0 = torch.empty((B, D), dtype=torch.float32, device=device)
    keep, wp, wb = _workspace(_lib.pf_gated_workspace_bytes(B, L, D, dt), workspace, device)
    _call(_lib.pf_gated_bwd, "pf_gated_bwd", device, (
        _ptr(X), *((0, 0) if X is None else _steps(X)), G.data_ptr(), *_steps(G), _ptr(h0), Y.data_ptr(), dY.data_ptr(), *_steps(dY),
        _ptr(dhL), dX.data_ptr(), dG.data_ptr(), dh0.data_ptr(), B, L, D, form, int(mix), dt, wp, wb, _stream_of(device, stream)))
    return dX, dG, dh0
