// C ABI of include/pf_layer.h: argument checks on the host, then the kernel launchers.
#include "../../include/pf_layer.h"
#include "pf_layer_internal.h"

#include <algorithm>
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

extern "C" int pf_head_norm_supported(int d, int rot, pf_dtype dt)
{
    return known(dt) && d >= 1 && rot >= 0 && rot <= d && rot % 2 == 0 && d <= 16 * pf::kHeadUnits && pf::head_units(d, rot) <= pf::kHeadUnits;
}

namespace {

pf_status heads_checks(const pf::Heads &a, bool backward, pf_norm_kind kind, pf_dtype dt)
{
    if (a.M < 0 || a.d <= 0 || a.rot < 0 || a.rot > a.d || a.rot % 2) return PF_ERR_SHAPE;
    if (a.side[0].H < 0 || a.side[1].H < 0 || a.far < 0) return PF_ERR_SHAPE;
    if (!pf_head_norm_supported(a.d, a.rot, dt) || (kind != PF_NORM_RMS && kind != PF_NORM_L2)) return PF_ERR_UNSUPPORTED;
    if ((long long)a.side[0].H + a.side[1].H > pf::kHeadsMost) return PF_ERR_UNSUPPORTED;
    const bool rows = a.M > 0;
    if (rows && a.rot && (!a.table || !a.positions)) return PF_ERR_NULL;
    for (const pf::HeadSide &s : a.side) {
        if (s.H == 0 || !rows) continue;
        if (!s.X || !s.Y || (backward && !s.dY)) return PF_ERR_NULL;
        if (s.xt < 0 || s.xh < 0 || s.dyt < 0 || s.dyh < 0) return PF_ERR_SHAPE;
    }
    if (!elements_aligned(dt, a.side[0].X, a.side[1].X, a.side[0].dY, a.side[1].dY) || reinterpret_cast<uintptr_t>(a.positions) % 4) return PF_ERR_ALIGN;
    if (!all_aligned(a.side[0].w, a.side[1].w, a.side[0].Y, a.side[1].Y, a.side[0].dw, a.side[1].dw, a.table, a.part)) return PF_ERR_ALIGN;
    return PF_OK;
}

}  // namespace

extern "C" pf_status pf_head_norm_fwd(const void *Q, long long qt, long long qh, const void *K, long long kt, long long kh,
                                      const void *wq, const void *wk, const float *table, int far, const int *positions, void *Yq,
                                      void *Yk, int M, int Hq, int Hk, int d, int rot, pf_norm_kind kind, int pairs, float eps,
                                      float q_scale, pf_dtype dt, pf_stream stream)
{
    pf::Heads a = {};
    a.side[0].X = Q, a.side[0].w = wq, a.side[0].Y = Yq, a.side[0].xt = qt, a.side[0].xh = qh, a.side[0].H = Hq, a.side[0].scale = q_scale;
    a.side[1].X = K, a.side[1].w = wk, a.side[1].Y = Yk, a.side[1].xt = kt, a.side[1].xh = kh, a.side[1].H = Hk, a.side[1].scale = 1.f;
    a.table = table, a.positions = positions, a.M = M, a.d = d, a.rot = rot, a.far = far, a.pairs = pairs != 0, a.l2 = kind == PF_NORM_L2, a.eps = eps;
    if (pf_status s = heads_checks(a, false, kind, dt)) return s;
    if (M == 0 || Hq + Hk == 0) return PF_OK;
    return launched(pf::launch_heads_fwd(a, dt == PF_BF16, on(stream)));
}

extern "C" size_t pf_head_norm_bwd_workspace_bytes(int M, int Hq, int Hk, int d, int rot)
{
    if (M <= 0 || Hq < 0 || Hk < 0 || (long long)Hq + Hk > pf::kHeadsMost || !pf_head_norm_supported(d, rot, PF_F32)) return 0;
    return (size_t)pf::heads_bwd_parts(M, Hq, Hk, d, rot) * d * sizeof(float);
}

extern "C" pf_status pf_head_norm_bwd(const void *Q, long long qt, long long qh, const void *K, long long kt, long long kh,
                                      const void *dYq, long long dyqt, long long dyqh, const void *dYk, long long dykt, long long dykh,
                                      const void *wq, const void *wk, const float *table, int far, const int *positions, void *dQ,
                                      void *dK, float *dwq, float *dwk, int M, int Hq, int Hk, int d, int rot, pf_norm_kind kind,
                                      int pairs, float eps, float q_scale, pf_dtype dt, void *workspace, size_t workspace_bytes,
                                      pf_stream stream)
{
    pf::Heads a = {};
    a.side[0] = {Q, wq, dYq, dQ, dwq, qt, qh, dyqt, dyqh, Hq, q_scale};
    a.side[1] = {K, wk, dYk, dK, dwk, kt, kh, dykt, dykh, Hk, 1.f};
    a.table = table, a.positions = positions, a.M = M, a.d = d, a.rot = rot, a.far = far, a.pairs = pairs != 0, a.l2 = kind == PF_NORM_L2, a.eps = eps;
    a.part = static_cast<float *>(workspace);
    if (pf_status s = heads_checks(a, true, kind, dt)) return s;
    const bool weights = dwq || dwk, rows = M > 0 && Hq + Hk > 0;
    if (weights && rows && (!workspace || workspace_bytes < pf_head_norm_bwd_workspace_bytes(M, Hq, Hk, d, rot))) return PF_ERR_WORKSPACE;
    if (!rows && !weights) return PF_OK;
    return launched(pf::launch_heads_bwd(a, dt == PF_BF16, on(stream)));
}

namespace {

bool gdelta_known(int Hk, int Hv, int dk, int dv, pf_dtype dt)
{
    return known(dt) && dk <= pf::kGDeltaWidest && dv <= pf::kGDeltaWidest && Hk >= 1 && Hv % Hk == 0;
}
pf_status gdelta_sizes(pf::GDelta &a, pf_dtype dt)
{
    if (a.N < 0 || a.L < 0 || a.Hk <= 0 || a.Hv <= 0 || a.dk <= 0 || a.dv <= 0 || a.Hv % a.Hk) return PF_ERR_SHAPE;
    if (a.L > 1 << 30 || !gdelta_known(a.Hk, a.Hv, a.dk, a.dv, dt)) return PF_ERR_UNSUPPORTED;
    // chunks, and threads of the kernels that have a workgroup for each of them and a head, or for 16 rows of a sequence's state, are counted in 32 bits
    const long long C = pf::kGDeltaChunk, some = a.N < a.L ? a.N : a.L;
    const long long per = (a.L + C - 1) / C, chunks = a.offsets ? (a.L + (C - 1) * some) / C : per * a.N;
    if (!pf::launch_holds((double)chunks * a.Hv, 512) || !pf::launch_holds((double)a.N * a.Hv * ((a.dv + 31) / 32 * 2), 768)) return PF_ERR_UNSUPPORTED;
    a.per = (int)per, a.chunks = (int)chunks;
    a.segments = pf::gdelta_segments(a);
    a.rows = a.offsets ? 0 : a.L;
    if (a.offsets) a.qb = a.kb = a.vb = a.gb = a.bb = a.ob = 0;      // (all in one row of tokens)
    return PF_OK;
}
// what both directions read
pf_status gdelta_inputs(const pf::GDelta &a, pf_dtype dt)
{
    if (a.chunks > 0 && (!a.Q || !a.K || !a.V || !a.G || !a.beta)) return PF_ERR_NULL;
    for (long long s : {a.qb, a.qt, a.qh, a.kb, a.kt, a.kh, a.vb, a.vt, a.vh, a.gb, a.gt, a.gh, a.bb, a.bt, a.bh, a.ob, a.ot, a.oh})
        if (s < 0) return PF_ERR_SHAPE;
    if (!elements_aligned(dt, a.Q, a.K, a.V, a.G, a.beta, a.dO) || reinterpret_cast<uintptr_t>(a.offsets) % 4) return PF_ERR_ALIGN;
    return PF_OK;
}

}  // namespace

extern "C" int pf_gated_delta_supported(int Hk, int Hv, int dk, int dv, pf_dtype dt)
{
    return dk >= 1 && dv >= 1 && Hv >= 1 && gdelta_known(Hk, Hv, dk, dv, dt);
}

extern "C" size_t pf_gated_delta_workspace_bytes(int N, int L, int Hk, int Hv, int dk, int dv, int packed, int backward, pf_dtype dt)
{
    pf::GDelta a = {};
    a.N = N, a.L = L, a.Hk = Hk, a.Hv = Hv, a.dk = dk, a.dv = dv;
    static const int some = 0;
    a.offsets = packed ? &some : nullptr;
    if (gdelta_sizes(a, dt) != PF_OK || a.chunks == 0) return 0;
    size_t bytes = pf::gdelta_workspace(a, backward != 0, nullptr);
    // fewer sequences are cut into more segments, or at all, and may take more (none from 29 on: each has 6 chains at least)
    for (int n = 1; n < N; ++n) {
        a.N = n;
        if (gdelta_sizes(a, dt) != PF_OK || a.segments == 1) break;
        bytes = std::max(bytes, pf::gdelta_workspace(a, backward != 0, nullptr));
    }
    return bytes;
}

extern "C" pf_status pf_gated_delta_fwd(const void *Q, long long qb, long long qt, long long qh, const void *K, long long kb, long long kt,
                                        long long kh, const void *V, long long vb, long long vt, long long vh, const void *G, long long gb,
                                        long long gt, long long gh, const void *beta, long long bb, long long bt, long long bh,
                                        const float *S0, const int *offsets, void *O, float *SL, int N, int L, int Hk, int Hv, int dk,
                                        int dv, pf_dtype dt, void *workspace, size_t workspace_bytes, pf_stream stream)
{
    pf::GDelta a = {};
    a.Q = Q, a.K = K, a.V = V, a.G = G, a.beta = beta, a.S0 = S0, a.offsets = offsets, a.O = O, a.SL = SL;
    a.qb = qb, a.qt = qt, a.qh = qh, a.kb = kb, a.kt = kt, a.kh = kh, a.vb = vb, a.vt = vt, a.vh = vh;
    a.gb = gb, a.gt = gt, a.gh = gh, a.bb = bb, a.bt = bt, a.bh = bh;
    a.N = N, a.L = L, a.Hk = Hk, a.Hv = Hv, a.dk = dk, a.dv = dv;
    if (pf_status s = gdelta_sizes(a, dt)) return s;
    if (N == 0) return PF_OK;
    if (pf_status s = gdelta_inputs(a, dt)) return s;
    if (a.chunks > 0 && !O) return PF_ERR_NULL;
    if (!all_aligned(S0, O, SL, workspace)) return PF_ERR_ALIGN;
    if (a.chunks == 0 && !SL) return PF_OK;
    if (a.chunks > 0 && (!workspace || workspace_bytes < pf::gdelta_workspace(a, false, nullptr))) return PF_ERR_WORKSPACE;
    if (a.chunks > 0) pf::gdelta_workspace(a, false, workspace);
    return launched(pf::launch_gdelta_fwd(a, dt == PF_BF16, on(stream)));
}

extern "C" pf_status pf_gated_delta_bwd(const void *Q, long long qb, long long qt, long long qh, const void *K, long long kb, long long kt,
                                        long long kh, const void *V, long long vb, long long vt, long long vh, const void *G, long long gb,
                                        long long gt, long long gh, const void *beta, long long bb, long long bt, long long bh,
                                        const void *dO, long long ob, long long ot, long long oh, const float *S0, const float *dSL,
                                        const int *offsets, void *dQ, void *dK, void *dV, void *dG, void *dbeta, float *dS0, int N, int L,
                                        int Hk, int Hv, int dk, int dv, pf_dtype dt, void *workspace, size_t workspace_bytes, pf_stream stream)
{
    pf::GDelta a = {};
    a.Q = Q, a.K = K, a.V = V, a.G = G, a.beta = beta, a.dO = dO, a.S0 = S0, a.dSL = dSL, a.offsets = offsets;
    a.dQ = dQ, a.dK = dK, a.dV = dV, a.dG = dG, a.dbeta = dbeta, a.dS0 = dS0;
    a.qb = qb, a.qt = qt, a.qh = qh, a.kb = kb, a.kt = kt, a.kh = kh, a.vb = vb, a.vt = vt, a.vh = vh;
    a.gb = gb, a.gt = gt, a.gh = gh, a.bb = bb, a.bt = bt, a.bh = bh, a.ob = ob, a.ot = ot, a.oh = oh;
    a.N = N, a.L = L, a.Hk = Hk, a.Hv = Hv, a.dk = dk, a.dv = dv;
    if (pf_status s = gdelta_sizes(a, dt)) return s;
    if (N == 0) return PF_OK;
    if (pf_status s = gdelta_inputs(a, dt)) return s;
    if (a.chunks > 0 && (!dO || !dQ || !dK || !dV || !dG || !dbeta)) return PF_ERR_NULL;
    if (!all_aligned(S0, dSL, dQ, dK, dV, dG, dbeta, dS0, workspace)) return PF_ERR_ALIGN;
    if (a.chunks == 0 && !dS0) return PF_OK;
    if (a.chunks > 0 && (!workspace || workspace_bytes < pf::gdelta_workspace(a, true, nullptr))) return PF_ERR_WORKSPACE;
    if (a.chunks > 0) pf::gdelta_workspace(a, true, workspace);
    return launched(pf::launch_gdelta_bwd(a, dt == PF_BF16, on(stream)));
}

extern "C" pf_status pf_gated_delta_step(const void *Q, long long qb, long long qh, const void *K, long long kb, long long kh, const void *V,
                                         long long vb, long long vh, const void *G, long long gb, long long gh, const void *beta,
                                         long long bb, long long bh, float *S, const int *slots, void *O, int B, int pool, int Hk, int Hv,
                                         int dk, int dv, pf_dtype dt, pf_stream stream)
{
    if (B < 0 || pool < 0 || Hk <= 0 || Hv <= 0 || dk <= 0 || dv <= 0 || Hv % Hk) return PF_ERR_SHAPE;
    if (!gdelta_known(Hk, Hv, dk, dv, dt)) return PF_ERR_UNSUPPORTED;
    if (B == 0) return PF_OK;
    if (!Q || !K || !V || !G || !beta || !O || (pool > 0 && !S)) return PF_ERR_NULL;
    for (long long s : {qb, qh, kb, kh, vb, vh, gb, gh, bb, bh})
        if (s < 0) return PF_ERR_SHAPE;
    if (!slots && pool < B) return PF_ERR_SHAPE;
    if (!elements_aligned(dt, Q, K, V, G, beta) || reinterpret_cast<uintptr_t>(slots) % 4 || !all_aligned(S, O)) return PF_ERR_ALIGN;
    return launched(pf::launch_gdelta_step({Q, K, V, G, beta, qb, qh, kb, kh, vb, vh, gb, gh, bb, bh, S, slots, O, B, pool, Hk, Hv, dk, dv},
                                           dt == PF_BF16, on(stream)));
}
