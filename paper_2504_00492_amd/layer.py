"""ctypes binding of include/pf_layer.h: the operators of a layer around the delta rule.  Argument marshalling only, as in
binding.py: every step of the computation runs in the HIP kernels of libpf_layer.so, PyTorch supplies device memory and the
stream, and without the library this module raises.

The functions without the pf_ prefix take torch tensors on the GPU, check them, allocate the outputs (and a workspace unless
one is handed in) and make one library call on the current stream of the tensors' device, or on `stream`, which all of them take.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

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
#
# A small call is bound by what happens here (a launch alone takes the host 3.4 us), so every tensor is looked at in as few
# steps as tell that it is right; _refuse finds out what is wrong with one that is not.

_BF, _F32, _E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
_DT = {_BF: PF_BF16, _F32: PF_F32}
_empty, _like, _stream, _current = torch.empty, torch.empty_like, torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _refuse(t, what, shape, dtype, index):
    if not t.is_cuda or t.get_device() != index:
        raise ValueError(f"{what} must be on cuda:{index}; there is no CPU path")
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    raise ValueError(f"{what} must be contiguous")


def _first(t, what, dims):
    """Type code and device index of the tensor that the others go by."""
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA (HIP) tensor; there is no CPU path")
    if t.dim() != dims:
        raise ValueError(f"{what} must have {('two', 'three')[dims - 2]} dimensions")
    dt = _DT.get(t.dtype)
    if dt is None:
        raise ValueError(f"{what} must be float32 or bfloat16")
    return dt, t.get_device()


def _dense(t, what, shape, dtype, index):
    """Address of a contiguous tensor of this shape and type, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or not t.is_contiguous():
        _refuse(t, what, shape, dtype, index)
    return t.data_ptr()


def _inner(t, what):
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the innermost dimension of {what} must be contiguous")


def _rows(t, what, shape, dtype, index):
    """Address and row stride of a matrix whose rows may lie apart (any stride serves where there is but one row)."""
    if t is None:
        return None, 0
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        _refuse(t, what, shape, dtype, index)
    if t.is_contiguous():
        return t.data_ptr(), shape[1]
    _inner(t, what)
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else max(shape[1], t.stride(0))


def _steps(t, what, shape, dtype, index):
    """Address, batch and token stride of [B, L, D] (where there is but one of them, what a dense array would have)."""
    if t is None:
        return None, 0, 0
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        _refuse(t, what, shape, dtype, index)
    B, L, D = shape
    if t.is_contiguous():
        return t.data_ptr(), L * D, D
    _inner(t, what)
    token = t.stride(1) if L > 1 else D
    return t.data_ptr(), t.stride(0) if B > 1 else L * token, token


def _byte_rows(M, K, device):
    """An uninitialised e4m3 matrix whose rows lie a multiple of 16 bytes apart."""
    ld = -(-K // 16) * 16
    q = _empty((M, ld), dtype=_E4, device=device)
    return q if ld == K else q[:, :K]


def _byte_matrix(t, what, shape, index):
    """Address and row stride of an e4m3 matrix, whose last row too must be held in whole 16 bytes."""
    if t.dtype is not _E4 or t.get_device() != index or t.shape != shape:
        _refuse(t, what, shape, _E4, index)
    rows, K = shape
    if K % 16 == 0 and t.is_contiguous():
        return t.data_ptr(), K
    _inner(t, what)
    whole = -(-K // 16) * 16
    ld = t.stride(0) if rows > 1 else max(whole, t.stride(0) // 16 * 16)
    if rows and t.storage_offset() + (rows - 1) * ld + whole > t.untyped_storage().nbytes():
        raise ValueError(f"the rows of {what} must be held in a multiple of 16 bytes")
    return t.data_ptr(), ld


def _same(t):
    """An uninitialised dense tensor of t's shape and type (0.5 us less than naming both, where t is dense itself)."""
    return _like(t) if t.is_contiguous() else _empty(t.shape, dtype=t.dtype, device=t.device)


def _workspace(need, given, device):
    """(tensor, address, bytes) of the workspace handed in, or of a new one; the tensor is kept until the call has been made."""
    if given is None:
        if not need:
            return None, None, 0
        given = _empty(need, dtype=torch.uint8, device=device)
    elif given.device != device:
        raise ValueError(f"workspace must be on {device}; there is no CPU path")
    elif not given.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return given, given.data_ptr(), given.numel() * given.element_size()


def _call(fn, name, index, *args):
    """One library call on the current stream of the tensors' device, with that device as the current one."""
    if _current() == index:
        st = fn(*args, _stream(index))
    else:
        with torch.cuda.device(index):
            st = fn(*args, _stream(index))
    if st != PF_OK:
        raise PfError(st, name)


def _on_stream(f):
    """f with an argument `stream` (a torch stream, or the handle of one; None: the current one).  The call's outputs and workspace
    come from that stream's memory, as if it had been made current: memory of another stream could still be in use there,
    or be handed out again there before the call is through.  What the call reads is the caller's to order and to keep until then, as
    with a current stream."""
    @functools.wraps(f)
    def with_stream(*args, stream=None, **kwargs):
        if stream is None:
            return f(*args, **kwargs)
        first = next((t for t in (*args, *kwargs.values()) if isinstance(t, torch.Tensor)), None)
        if first is None:
            raise ValueError("there is no tensor whose device the stream could be of")
        if not first.is_cuda:
            return f(*args, **kwargs)      # (which says what is wrong with it)
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, first.device) if stream else torch.cuda.default_stream(first.device)
        elif stream.device != first.device:
            raise ValueError(f"stream must be one of {first.device}")
        with torch.cuda.stream(stream):
            return f(*args, **kwargs)
    return with_stream


@_on_stream
def norm_fwd(X, w=None, R=None, *, eps, y: bool = True, fp8: bool = False, inplace: bool = False):
    """Root-mean-square norm of the rows of X + R (pf_norm_fwd).  X, R [M, D] (float32 or bfloat16, rows may lie apart), w [D]
    of the same type.  Returns (S, Y, Q, scale): S the stored sum (X itself without R; R's own memory with inplace, which
    asks for a contiguous R), Y the norm (None with y=False), Q and scale the norm in 8 bits (None unless fp8)."""
    dt, index = _first(X, "X", 2)
    shape, dtype = X.shape, X.dtype
    M, D = shape
    xp, ldx = _rows(X, "X", shape, dtype, index)
    rp, ldr = _rows(R, "R", shape, dtype, index)
    wp = _dense(w, "w", (D,), dtype, index)
    if not (y or fp8):
        raise ValueError("neither y nor fp8 is wanted")
    if inplace:
        if R is None:
            raise ValueError("inplace needs R")
        _dense(R, "R", shape, dtype, index)
    device = X.device
    S, sp = X, None
    if R is not None:
        S = R if inplace else _same(X)
        sp = S.data_ptr()
    Y = yp = Q = qp = scale = cp = None
    if y:
        Y = _same(X)
        yp = Y.data_ptr()
    if fp8:
        Q, scale = _byte_rows(M, D, device), _empty((-(-D // 128), M), dtype=_F32, device=device)
        qp, cp = Q.data_ptr(), scale.data_ptr()
    _call(_lib.pf_norm_fwd, "pf_norm_fwd", index, xp, ldx, rp, ldr, wp, sp, yp, qp, -(-D // 16) * 16, cp, M, D, eps, dt)
    return S, Y, Q, scale


@_on_stream
def norm_bwd(S, dY, w=None, dS=None, *, eps, want_dw: bool = True, workspace=None):
    """Backward of norm_fwd (pf_norm_bwd): S the stored sum, dY the gradient of the norm, dS that of the sum past the norm
    (None: none).  Returns (dX, dw): dX [M, D] in the inputs' type, dw [D] in float32 (None unless wanted)."""
    dt, index = _first(S, "S", 2)
    shape, dtype, device = S.shape, S.dtype, S.device
    M, D = shape
    sp, lds = _rows(S, "S", shape, dtype, index)
    yp, ldy = _rows(dY, "dY", shape, dtype, index)
    rp, ldr = _rows(dS, "dS", shape, dtype, index)
    wp = _dense(w, "w", (D,), dtype, index)
    dX = _same(S)
    dw = dp = keep = kp = None
    kb = 0
    if want_dw:
        dw = _empty(D, dtype=_F32, device=device)
        dp = dw.data_ptr()
        keep, kp, kb = _workspace(_lib.pf_norm_bwd_workspace_bytes(M, D) if workspace is None else 0, workspace, device)
    _call(_lib.pf_norm_bwd, "pf_norm_bwd", index, sp, lds, wp, yp, ldy, rp, ldr, dX.data_ptr(), dp, M, D, eps, dt, kp, kb)
    return dX, dw


@_on_stream
def quant_fp8(X, *, rows: int = 1, plain: bool = True, transposed: bool = False):
    """X [M, K] (float32 or bfloat16, rows may lie apart) in 8 bits (pf_quant_fp8), with a scale for each row and 128 columns
    (rows=1) or each 128 x 128 (rows=128).  Returns (Q, scale, QT, scaleT); Q and scale are None with plain=False, QT and
    scaleT (the transposed matrix, its blocks along its own rows) unless transposed."""
    dt, index = _first(X, "X", 2)
    M, K = X.shape
    xp, ldx = _rows(X, "X", X.shape, X.dtype, index)
    if rows not in (1, 128):
        raise ValueError("rows must be 1 or 128")
    if not (plain or transposed):
        raise ValueError("neither plain nor transposed is wanted")
    device = X.device
    Q = qp = scale = sp = QT = tp = scaleT = up = None
    if plain:
        Q = _byte_rows(M, K, device)
        scale = _empty((-(-K // 128), M if rows == 1 else -(-M // 128)), dtype=_F32, device=device)
        qp, sp = Q.data_ptr(), scale.data_ptr()
    if transposed:
        QT = _byte_rows(K, M, device)
        scaleT = _empty((-(-M // 128), K if rows == 1 else -(-K // 128)), dtype=_F32, device=device)
        tp, up = QT.data_ptr(), scaleT.data_ptr()
    _call(_lib.pf_quant_fp8, "pf_quant_fp8", index, xp, ldx, qp, -(-K // 16) * 16, sp, tp, -(-M // 16) * 16, up, M, K, rows, dt)
    return Q, scale, QT, scaleT


@_on_stream
def matmul_fp8(A, sa, B, sb, *, b_rows: int = 128, out_dtype=_BF, workspace=None):
    """C [M, N] = A [M, K] times B [N, K] transposed, both e4m3 with scales (pf_matmul_fp8): sa [ceil(K/128), M], sb
    [ceil(K/128), N] (b_rows=1) or [ceil(K/128), ceil(N/128)] (b_rows=128).  Rows of A and B lie a multiple of 16 bytes apart,
    as quant_fp8 and norm_fwd lay them.  out_dtype: bfloat16 or float32, which chooses the sums too: float32 sums of exact products, or those
    of the 8-bit instruction, which drops of eight products what lies 2^-13 below the largest."""
    if not A.is_cuda:
        raise ValueError("A must be a CUDA (HIP) tensor; there is no CPU path")
    if A.dim() != 2 or B.dim() != 2:
        raise ValueError("A and B must have two dimensions")
    if b_rows not in (1, 128):
        raise ValueError("b_rows must be 1 or 128")
    dt = _DT.get(out_dtype)
    if dt is None:
        raise ValueError("out_dtype must be float32 or bfloat16")
    index, device = A.get_device(), A.device
    M, K = A.shape
    N = B.shape[0]
    nk = -(-K // 128)
    ap, lda = _byte_matrix(A, "A", (M, K), index)
    bp, ldb = _byte_matrix(B, "B", (N, K), index)
    sap = _dense(sa, "sa", (nk, M), _F32, index)
    sbp = _dense(sb, "sb", (nk, N if b_rows == 1 else -(-N // 128)), _F32, index)
    C = _empty((M, N), dtype=out_dtype, device=device)
    # (16 rows at most never need a workspace)
    keep, kp, kb = _workspace(_lib.pf_matmul_fp8_workspace_bytes(M, N, K, b_rows) if workspace is None and M > 16 else 0, workspace, device)
    _call(_lib.pf_matmul_fp8, "pf_matmul_fp8", index, ap, lda, sap, bp, ldb, sbp, b_rows, C.data_ptr(), N, M, N, K, dt, kp, kb)
    return C


def _gate_of(gate):
    if gate not in GATES:
        raise ValueError(f"gate must be one of {', '.join(GATES)}")
    return GATES[gate]


@_on_stream
def gated_fwd(X, G, h0=None, *, gate: str = "log", mix: bool = False, workspace=None):
    """The gated linear recurrence h_t = a_t h_{t-1} + b_t (pf_gated_fwd): a = G, exp(G) or its sigmoid by gate ("value",
    "log", "logit"), b = X, or (1 - a) X with mix.  X, G [B, L, D] (float32 or bfloat16, tokens and sequences may lie apart or in the
    other order), h0 [B, D] float32 or None.  Returns (Y [B, L, D], h_L [B, D] float32)."""
    dt, index = _first(X, "X", 3)
    form = _gate_of(gate)
    shape, dtype, device = X.shape, X.dtype, X.device
    B, L, D = shape
    x = _steps(X, "X", shape, dtype, index)
    g = _steps(G, "G", shape, dtype, index)
    hp = _dense(h0, "h0", (B, D), _F32, index)
    Y, hL = _same(X), _empty((B, D), dtype=_F32, device=device) if h0 is None else _like(h0)
    # (16 tokens at most never need a workspace)
    keep, kp, kb = _workspace(_lib.pf_gated_workspace_bytes(B, L, D, dt) if workspace is None and L > 16 else 0, workspace, device)
    _call(_lib.pf_gated_fwd, "pf_gated_fwd", index, *x, *g, hp, Y.data_ptr(), hL.data_ptr(), B, L, D, form, bool(mix), dt, kp, kb)
    return Y, hL


@_on_stream
def gated_bwd(X, G, Y, dY, h0=None, dhL=None, *, gate: str = "log", mix: bool = False, workspace=None):
    """Backward of gated_fwd (pf_gated_bwd) from what it was given and returned (X may be None without mix), dY the gradient of
    Y, dhL that of h_L (float32, None: none).  Returns (dX, dG, dh0)."""
    dt, index = _first(G, "G", 3)
    form = _gate_of(gate)
    if mix and X is None:
        raise ValueError("mix needs X")
    shape, dtype, device = G.shape, G.dtype, G.device
    B, L, D = shape
    x = _steps(X, "X", shape, dtype, index)
    g = _steps(G, "G", shape, dtype, index)
    yp = _dense(Y, "Y", shape, dtype, index)
    dy = _steps(dY, "dY", shape, dtype, index)
    hp, ep = _dense(h0, "h0", (B, D), _F32, index), _dense(dhL, "dhL", (B, D), _F32, index)
    dX, dG = _same(G), _same(G)
    dh0 = _empty((B, D), dtype=_F32, device=device) if h0 is None else _like(h0)
    keep, kp, kb = _workspace(_lib.pf_gated_workspace_bytes(B, L, D, dt) if workspace is None and L > 16 else 0, workspace, device)
    _call(_lib.pf_gated_bwd, "pf_gated_bwd", index, *x, *g, hp, yp, *dy, ep, dX.data_ptr(), dG.data_ptr(), dh0.data_ptr(), B, L, D,
          form, bool(mix), dt, kp, kb)
    return dX, dG, dh0
