"""Host-side checks of include/pf_layer.h: the library exports what the header declares, and every argument check returns
its code before anything is launched (no GPU needed)."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2504_00492_amd", "libpf_layer.so")
P = 0x1000          # an address that no check follows
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def layer():
    if not os.path.exists(LIB):
        from paper_2504_00492_amd import build
        build.build_library()
    from paper_2504_00492_amd import layer
    return layer


def test_header_symbols_are_exported(layer):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "pf_layer.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(pf_[a-z0-9_]+)\s*\(", text)))
    lib = ctypes.CDLL(LIB)
    assert names == sorted(layer.EXPORTS) and all(hasattr(lib, n) for n in names)


def test_header_is_plain_c(layer, tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "pf_layer.h"\nint main(void) { return pf_norm_supported(4096, PF_BF16) != 1; }\n')
    exe, where = str(tmp_path / "t"), os.path.dirname(LIB)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), LIB, "-o", exe,
                    "-Wl,-rpath," + where, "-Wl,--allow-shlib-undefined"], check=True)
    assert subprocess.run([exe]).returncode == 0


def _norm_fwd(pf, **k):
    a = dict(X=P, ldx=64, R=P, ldr=64, w=P, S=P, Y=P, Q=P, ldq=64, scale=P, M=4, D=64, eps=1e-5, dt=BF16, stream=0) | k
    return pf.pf_norm_fwd(**a)


def _norm_bwd(pf, **k):
    a = dict(S=P, lds=64, w=P, dY=P, lddy=64, dS=P, ldds=64, dX=P, dw=P, M=4, D=64, eps=1e-5, dt=BF16, workspace=P,
             workspace_bytes=1 << 30, stream=0) | k
    return pf.pf_norm_bwd(**a)


def _quant(pf, **k):
    a = dict(X=P, ldx=64, Q=P, ldq=64, scale=P, QT=P, ldqt=16, scaleT=P, M=4, K=64, rows=1, dt=BF16, stream=0) | k
    return pf.pf_quant_fp8(**a)


def _matmul(pf, **k):
    a = dict(A=P, lda=64, sa=P, B=P, ldb=64, sb=P, b_rows=128, C=P, ldc=8, M=4, N=8, K=64, dt=BF16, workspace=P,
             workspace_bytes=1 << 40, stream=0) | k
    return pf.pf_matmul_fp8(**a)


def _gated_fwd(pf, **k):
    a = dict(X=P, xb=64, xt=8, G=P, gb=64, gt=8, h0=P, Y=P, hL=P, B=2, L=8, D=8, gate=1, mix=0, dt=BF16, workspace=P,
             workspace_bytes=1 << 40, stream=0) | k
    return pf.pf_gated_fwd(**a)


def _gated_bwd(pf, **k):
    a = dict(X=P, xb=64, xt=8, G=P, gb=64, gt=8, h0=P, Y=P, dY=P, dyb=64, dyt=8, dhL=P, dX=P, dG=P, dh0=P, B=2, L=8, D=8,
             gate=1, mix=1, dt=BF16, workspace=P, workspace_bytes=1 << 40, stream=0) | k
    return pf.pf_gated_bwd(**a)


NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


@pytest.mark.parametrize("call,wrong,status", [
    (_norm_fwd, dict(X=None), NULL), (_norm_fwd, dict(Y=None, Q=None), NULL), (_norm_fwd, dict(scale=None), NULL),
    (_norm_fwd, dict(M=-1), SHAPE), (_norm_fwd, dict(D=0), SHAPE), (_norm_fwd, dict(ldx=63), SHAPE),
    (_norm_fwd, dict(ldr=63), SHAPE), (_norm_fwd, dict(ldq=72), SHAPE), (_norm_fwd, dict(ldq=48), SHAPE),
    (_norm_fwd, dict(D=16385, ldx=20000, ldr=20000, ldq=20000), UNSUPPORTED), (_norm_fwd, dict(dt=2), UNSUPPORTED),
    (_norm_fwd, dict(X=P + 1), ALIGN), (_norm_fwd, dict(w=P + 2), ALIGN), (_norm_fwd, dict(Q=P + 8), ALIGN), (_norm_fwd, dict(scale=P + 4), ALIGN),
    (_norm_bwd, dict(S=None), NULL), (_norm_bwd, dict(dY=None), NULL), (_norm_bwd, dict(dX=None), NULL),
    (_norm_bwd, dict(lddy=63), SHAPE), (_norm_bwd, dict(ldds=63), SHAPE), (_norm_bwd, dict(lds=8), SHAPE),
    (_norm_bwd, dict(dt=-1), UNSUPPORTED), (_norm_bwd, dict(dw=P + 4), ALIGN),
    (_norm_bwd, dict(workspace=None), WORKSPACE), (_norm_bwd, dict(workspace_bytes=64), WORKSPACE),
    (_quant, dict(X=None), NULL), (_quant, dict(Q=None, QT=None), NULL), (_quant, dict(scaleT=None), NULL),
    (_quant, dict(scale=None), NULL), (_quant, dict(M=-1), SHAPE), (_quant, dict(ldx=63), SHAPE), (_quant, dict(ldq=65), SHAPE),
    (_quant, dict(ldqt=4), SHAPE), (_quant, dict(ldqt=0), SHAPE), (_quant, dict(rows=64), UNSUPPORTED),
    (_quant, dict(dt=7), UNSUPPORTED), (_quant, dict(QT=P + 1), ALIGN),
    (_matmul, dict(A=None), NULL), (_matmul, dict(sa=None), NULL), (_matmul, dict(sb=None), NULL), (_matmul, dict(C=None), NULL),
    (_matmul, dict(K=0), SHAPE), (_matmul, dict(N=-1), SHAPE), (_matmul, dict(lda=72), SHAPE), (_matmul, dict(ldb=48), SHAPE),
    (_matmul, dict(ldc=7), SHAPE), (_matmul, dict(b_rows=2), UNSUPPORTED), (_matmul, dict(dt=2), UNSUPPORTED),
    (_matmul, dict(B=P + 8), ALIGN), (_matmul, dict(C=P + 2), ALIGN),
    (_gated_fwd, dict(X=None), NULL), (_gated_fwd, dict(G=None), NULL), (_gated_fwd, dict(Y=None), NULL),
    (_gated_fwd, dict(B=-1), SHAPE), (_gated_fwd, dict(L=-1), SHAPE), (_gated_fwd, dict(D=0), SHAPE), (_gated_fwd, dict(xt=-8), SHAPE),
    (_gated_fwd, dict(gate=3), UNSUPPORTED), (_gated_fwd, dict(L=(1 << 30) + 1), UNSUPPORTED), (_gated_fwd, dict(dt=2), UNSUPPORTED), (_gated_fwd, dict(h0=P + 4), ALIGN),
    (_gated_bwd, dict(X=None), NULL), (_gated_bwd, dict(Y=None), NULL), (_gated_bwd, dict(dY=None), NULL),
    (_gated_bwd, dict(dG=None), NULL), (_gated_bwd, dict(dyb=-1), SHAPE), (_gated_bwd, dict(gate=-1), UNSUPPORTED),
    (_gated_bwd, dict(dX=P + 2), ALIGN), (_gated_fwd, dict(G=P + 1), ALIGN)])
def test_refusals(layer, call, wrong, status):
    assert call(layer, **wrong) == status


@pytest.mark.parametrize("call,sizes", [
    (_quant, dict(M=(1 << 31) - 1, K=640, ldx=640, ldq=640, ldqt=1 << 31)),
    (_matmul, dict(M=1, N=(1 << 31) - 1, ldc=1 << 31)), (_matmul, dict(M=(1 << 31) - 1, N=272, ldc=272)),
    (_matmul, dict(M=(1 << 31) - 1, N=272, ldc=272, dt=F32)), (_matmul, dict(M=1 << 23, N=2, ldb=1 << 24)),
    (_gated_fwd, dict(B=1 << 26, L=1, D=1)), (_gated_fwd, dict(B=1 << 23, L=20, D=1)), (_gated_fwd, dict(B=(1 << 31) - 1, L=0, D=1 << 20)),
    (_gated_bwd, dict(B=2, L=1 << 30, D=1)), (_gated_bwd, dict(B=1 << 20, L=17, D=1 << 20))])
def test_more_than_a_launch_holds(layer, call, sizes):
    """Refused on the host, before any work."""
    assert call(layer, **sizes) == UNSUPPORTED



def test_workspace_too_small(layer):
    need = layer.pf_gated_workspace_bytes(1, 65536, 4096, BF16)
    if need:
        big = dict(B=1, L=65536, D=4096, xt=4096, gt=4096, dyt=4096)
        fwd = {k: v for k, v in big.items() if k != "dyt"}
        for call, k in ((_gated_fwd, fwd), (_gated_bwd, big)):
            assert call(layer, **k, workspace_bytes=need - 1) == WORKSPACE
            assert call(layer, **k, workspace=None) == WORKSPACE
    sizes = [(m, n, k) for m in (1, 16, 100, 512, 2048) for n in (128, 1000, 4096) for k in (128, 4096, 8192)]
    m, n, k = max(sizes, key=lambda s: layer.pf_matmul_fp8_workspace_bytes(*s, 128))
    need = layer.pf_matmul_fp8_workspace_bytes(m, n, k, 128)
    if need:
        a = dict(M=m, N=n, K=k, lda=k, ldb=k, ldc=n)
        assert _matmul(layer, **a, workspace_bytes=need - 1) == WORKSPACE
        assert _matmul(layer, **a, workspace=None) == WORKSPACE


def test_nothing_to_do(layer):
    """Empty calls return at once, with no pointer looked at."""
    none = dict.fromkeys(("X", "R", "w", "S", "Y", "Q", "scale"))
    assert _norm_fwd(layer, M=0, **none) == 0
    assert _norm_bwd(layer, M=0, S=None, w=None, dY=None, dS=None, dX=None, dw=None, workspace=None) == 0
    assert _quant(layer, M=0, X=None) == 0 and _quant(layer, K=0, X=None) == 0
    assert _matmul(layer, M=0, A=None) == 0 and _matmul(layer, N=0, A=None) == 0
    assert _gated_fwd(layer, B=0, X=None) == 0 and _gated_bwd(layer, B=0, X=None) == 0
    assert _gated_fwd(layer, L=0, X=None, G=None, Y=None, hL=None) == 0
    assert _gated_bwd(layer, L=0, G=None, dh0=None) == 0
    assert layer.pf_norm_bwd_workspace_bytes(0, 64) == 0 and layer.pf_gated_workspace_bytes(1, 0, 64, BF16) == 0
    assert layer.pf_matmul_fp8_workspace_bytes(0, 1, 1, 1) == 0


def test_small_calls_need_no_workspace(layer):
    for n in (1, 2, 15, 16):
        for wide in (1, 100, 4096, 20544):
            assert layer.pf_matmul_fp8_workspace_bytes(n, wide, 8192, 1) == layer.pf_matmul_fp8_workspace_bytes(n, wide, 8192, 128) == 0
            assert layer.pf_gated_workspace_bytes(7, n, wide, BF16) == layer.pf_gated_workspace_bytes(7, n, wide, F32) == 0


def test_workspace_is_bounded(layer):
    for M in (1, 7, 4096, 10**6):
        for D in (1, 128, 4096, 16384):
            assert 4 * D <= layer.pf_norm_bwd_workspace_bytes(M, D) <= 1 << 26
    assert [layer.pf_norm_supported(D, BF16) for D in (0, 1, 16384, 16385)] == [0, 1, 1, 0]
    assert layer.pf_norm_supported(64, 2) == 0


def test_tensor_checks(layer):
    """The functions on tensors say what is wrong with an argument; there is no CPU path."""
    import torch
    x = torch.zeros(4, 64)
    for call in (lambda: layer.norm_fwd(x, eps=0.), lambda: layer.norm_bwd(x, x, eps=0.), lambda: layer.quant_fp8(x),
                 lambda: layer.matmul_fp8(x, x, x, x), lambda: layer.gated_fwd(x[None], x[None]),
                 lambda: layer.gated_bwd(None, x[None], x[None], x[None])):
        with pytest.raises(ValueError, match="no CPU path"):
            call()
