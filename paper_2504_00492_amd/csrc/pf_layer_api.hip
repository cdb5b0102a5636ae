// C ABI of include/pf_layer.h: argument checks on the host, then the kernel launchers.
#include "../../include/pf_layer.h"
#include "pf_layer_internal.h"

#include <limits.h>

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
template <typename... P> bool all_aligned(P... p) { return (aligned16(p) && ...); }
// inputs with strides need their elements' alignment only: the kernels take wide loads where address and strides allow them
template <typename... P> bool elements_aligned(pf_dtype dt, P... p)
{
    return ((reinterpret_cast<uintptr_t>(p) % (dt == PF_F32 ? 4 : 2) == 0) && ...);
}
inline bool known(pf_dtype dt) { return dt == PF_F32 || dt == PF_BF16; }
inline pf_status launched(hipError_t e)
{
    return e == hipSuccess ? PF_OK : e == hipErrorInvalidConfiguration ? PF_ERR_UNSUPPORTED : PF_ERR_LAUNCH;
}
inline hipStream_t on(pf_stream s) { return static_cast<hipStream_t>(s); }

}  // namespace

extern "C" int pf_norm_supported(int D, pf_dtype dt) { return known(dt) && D >= 1 && D <= pf::kNormWidest; }

extern "C" pf_status pf_norm_fwd(const void *X, long long ldx, const void *R, long long ldr, const void *w, void *S, void *Y,
                                 void *Q, long long ldq, float *scale, int M, int D, float eps, pf_dtype dt, pf_stream stream)
{
    if (M < 0 || D <= 0) return PF_ERR_SHAPE;
    if (!pf_norm_supported(D, dt)) return PF_ERR_UNSUPPORTED;
    if (M == 0) return PF_OK;
    if (!X || (!Y && !Q) || (Q && !scale)) return PF_ERR_NULL;
    if (ldx < D || (R && ldr < D) || (Q && (ldq < D || ldq % 16))) return PF_ERR_SHAPE;
    if (!elements_aligned(dt, X, R) || !all_aligned(w, S, Y, Q, scale)) return PF_ERR_ALIGN;
    return launched(pf::launch_norm_fwd({X, R, w, S, Y, Q, scale, ldx, ldr, ldq, M, D, eps}, dt == PF_BF16, on(stream)));
}

extern "C" size_t pf_norm_bwd_workspace_bytes(int M, int D)
{
    if (M <= 0 || D <= 0 || D > pf::kNormWidest) return 0;
    return (size_t)pf::norm_bwd_parts(M, D) * D * sizeof(float);
}

extern "C" pf_status pf_norm_bwd(const void *S, long long lds, const void *w, const void *dY, long long lddy, const void *dS,
                                 long long ldds, void *dX, float *dw, int M, int D, float eps, pf_dtype dt, void *workspace,
                                 size_t workspace_bytes, pf_stream stream)
{
    if (M < 0 || D <= 0) return PF_ERR_SHAPE;
    if (!pf_norm_supported(D, dt)) return PF_ERR_UNSUPPORTED;
    if (M > 0 && (!S || !dY || !dX)) return PF_ERR_NULL;
    if (M > 0 && (lds < D || lddy < D || (dS && ldds < D))) return PF_ERR_SHAPE;
    if (!elements_aligned(dt, S, dY, dS) || !all_aligned(w, dX, dw, workspace)) return PF_ERR_ALIGN;
    if (dw && M > 0 && (!workspace || workspace_bytes < pf_norm_bwd_workspace_bytes(M, D))) return PF_ERR_WORKSPACE;
    if (M == 0 && !dw) return PF_OK;
    return launched(pf::launch_norm_bwd({S, w, dY, dS, dX, dw, static_cast<float *>(workspace), lds, lddy, ldds, M, D, eps},
                                        dt == PF_BF16, on(stream)));
}

extern "C" pf_status pf_quant_fp8(const void *X, long long ldx, void *Q, long long ldq, float *scale, void *QT, long long ldqt,
                                  float *scaleT, int M, int K, int rows, pf_dtype dt, pf_stream stream)
{
    if (M < 0 || K < 0) return PF_ERR_SHAPE;
    if (!known(dt) || (rows != 1 && rows != 128)) return PF_ERR_UNSUPPORTED;
    if (M == 0 || K == 0) return PF_OK;
    if (!X || (!Q && !QT) || (Q && !scale) || (QT && !scaleT)) return PF_ERR_NULL;
    if (ldx < K || (Q && (ldq < K || ldq % 16)) || (QT && (ldqt < M || ldqt % 16))) return PF_ERR_SHAPE;
    if (!elements_aligned(dt, X) || !all_aligned(Q, scale, QT, scaleT)) return PF_ERR_ALIGN;
    return launched(pf::launch_quant({X, Q, QT, scale, scaleT, ldx, ldq, ldqt, M, K, rows}, dt == PF_BF16, on(stream)));
}

// columns of a row are counted in 32 bits, in whole blocks of 128
static constexpr int kDeepest = INT_MAX - 127;

extern "C" size_t pf_matmul_fp8_workspace_bytes(int M, int N, int K, int b_rows)
{
    if (M <= 0 || N <= 0 || K <= 0 || K > kDeepest || (b_rows != 1 && b_rows != 128)) return 0;
    return pf::matmul_workspace_bytes(M, N, K, b_rows);
}

extern "C" pf_status pf_matmul_fp8(const void *A, long long lda, const float *sa, const void *B, long long ldb, const float *sb,
                                   int b_rows, void *C, long long ldc, int M, int N, int K, pf_dtype dt, void *workspace,
                                   size_t workspace_bytes, pf_stream stream)
{
    if (M < 0 || N < 0 || K <= 0) return PF_ERR_SHAPE;
    if (!known(dt) || (b_rows != 1 && b_rows != 128) || K > kDeepest) return PF_ERR_UNSUPPORTED;
    if (M == 0 || N == 0) return PF_OK;
    if (!A || !sa || !B || !sb || !C) return PF_ERR_NULL;
    if (lda < K || ldb < K || lda % 16 || ldb % 16 || ldc < N) return PF_ERR_SHAPE;
    if (!all_aligned(A, sa, B, sb, C, workspace)) return PF_ERR_ALIGN;
    const size_t need = pf_matmul_fp8_workspace_bytes(M, N, K, b_rows);
    if (need && (!workspace || workspace_bytes < need)) return PF_ERR_WORKSPACE;
    return launched(pf::launch_matmul({A, B, sa, sb, C, static_cast<float *>(workspace), lda, ldb, ldc, M, N, K, b_rows},
                                      dt == PF_BF16, on(stream)));
}

extern "C" size_t pf_gated_workspace_bytes(int B, int L, int D, pf_dtype dt)
{
    if (B <= 0 || L <= 0 || D <= 0 || !known(dt)) return 0;
    return pf::gated_workspace_bytes(B, L, D, dt == PF_BF16);
}

namespace {

pf_status gated_checks(int B, int L, int D, pf_gate gate, pf_dtype dt)
{
    if (B < 0 || L < 0 || D <= 0) return PF_ERR_SHAPE;
    if (L > 1 << 30 || !known(dt) || (gate != PF_GATE_VALUE && gate != PF_GATE_LOG && gate != PF_GATE_LOGIT)) return PF_ERR_UNSUPPORTED;
    return PF_OK;
}
pf_status gated_workspace(int B, int L, int D, pf_dtype dt, const void *workspace, size_t workspace_bytes)
{
    const size_t need = pf_gated_workspace_bytes(B, L, D, dt);
    return need && (!workspace || workspace_bytes < need) ? PF_ERR_WORKSPACE : PF_OK;
}

}  // namespace

extern "C" pf_status pf_gated_fwd(const void *X, long long xb, long long xt, const void *G, long long gb, long long gt,
                                  const float *h0, void *Y, float *hL, int B, int L, int D, pf_gate gate, int mix, pf_dtype dt,
                                  void *workspace, size_t workspace_bytes, pf_stream stream)
{
    if (pf_status s = gated_checks(B, L, D, gate, dt)) return s;
    if (B == 0) return PF_OK;
    if (L > 0 && (!X || !G || !Y)) return PF_ERR_NULL;
    if (xb < 0 || xt < 0 || gb < 0 || gt < 0) return PF_ERR_SHAPE;
    if (!elements_aligned(dt, X, G) || !all_aligned(h0, Y, hL, workspace)) return PF_ERR_ALIGN;
    if (pf_status s = gated_workspace(B, L, D, dt, workspace, workspace_bytes)) return s;
    if (L == 0 && !hL) return PF_OK;
    pf::Gated a = {};
    a.X = X, a.G = G, a.h0 = h0, a.Y = Y, a.hL = hL, a.work = workspace;
    a.xb = xb, a.xt = xt, a.gb = gb, a.gt = gt;
    a.B = B, a.L = L, a.D = D, a.gate = gate, a.mix = mix != 0;
    return launched(pf::launch_gated_fwd(a, dt == PF_BF16, on(stream)));
}

extern "C" pf_status pf_gated_bwd(const void *X, long long xb, long long xt, const void *G, long long gb, long long gt,
                                  const float *h0, const void *Y, const void *dY, long long dyb, long long dyt, const float *dhL,
                                  void *dX, void *dG, float *dh0, int B, int L, int D, pf_gate gate, int mix, pf_dtype dt,
                                  void *workspace, size_t workspace_bytes, pf_stream stream)
{
    if (pf_status s = gated_checks(B, L, D, gate, dt)) return s;
    if (B == 0) return PF_OK;
    if (L > 0 && ((mix && !X) || !G || !Y || !dY || !dX || !dG)) return PF_ERR_NULL;
    if (xb < 0 || xt < 0 || gb < 0 || gt < 0 || dyb < 0 || dyt < 0) return PF_ERR_SHAPE;
    if (!elements_aligned(dt, X, G, dY) || !all_aligned(h0, Y, dhL, dX, dG, dh0, workspace)) return PF_ERR_ALIGN;
    if (pf_status s = gated_workspace(B, L, D, dt, workspace, workspace_bytes)) return s;
    if (L == 0 && !dh0) return PF_OK;
    pf::Gated a = {};
    a.X = mix ? X : nullptr, a.G = G, a.h0 = h0, a.Yin = Y, a.dY = dY, a.dhL = dhL, a.dX = dX, a.dG = dG, a.dh0 = dh0;
    a.work = workspace;
    a.xb = xb, a.xt = xt, a.gb = gb, a.gt = gt, a.dyb = dyb, a.dyt = dyt;
    a.B = B, a.L = L, a.D = D, a.gate = gate, a.mix = mix != 0;
    return launched(pf::launch_gated_bwd(a, dt == PF_BF16, on(stream)));
}
