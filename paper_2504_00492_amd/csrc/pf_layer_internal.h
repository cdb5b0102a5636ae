// Host-side launchers behind the C ABI of include/pf_layer.h.  Each returns the HIP status of its launches; none of them
// allocates, frees or synchronises.
#pragma once
#include "pf_internal.h"

namespace pf {

// A launch holds fewer than 2^32 threads; a launcher that would need more returns hipErrorInvalidConfiguration before it launches anything.
inline bool launch_holds(double groups, int threads) { return groups * threads < 4294967296.0; }


// ---- root-mean-square norm (pf_norm.hip)
constexpr int kNormWidest = 16384;
struct NormFwd {
    const void *X, *R, *w;
    void *S, *Y, *Q;
    float *scale;
    long long ldx, ldr, ldq;
    int M, D;
    float eps;
};
hipError_t launch_norm_fwd(const NormFwd &a, bool is_bf16, hipStream_t stream);
struct NormBwd {
    const void *S, *w, *dY, *dS;
    void *dX;
    float *dw, *part;      // part [norm_bwd_parts(M, D)][D]
    long long lds, lddy, ldds;
    int M, D;
    float eps;
};
int norm_bwd_parts(int M, int D);
hipError_t launch_norm_bwd(const NormBwd &a, bool is_bf16, hipStream_t stream);

// ---- matrices in 8 bits (pf_quant.hip)
struct Quant {
    const void *X;
    void *Q, *QT;
    float *scale, *scaleT;
    long long ldx, ldq, ldqt;
    int M, K, rows;
};
hipError_t launch_quant(const Quant &a, bool is_bf16, hipStream_t stream);

// ---- product of matrices in 8 bits (pf_matmul.hip)
struct Matmul {
    const void *A, *B;
    const float *sa, *sb;
    void *C;
    float *part;
    long long lda, ldb, ldc;
    int M, N, K, b_rows;
    long long sb_ld;      // of the scales of B: set by launch_matmul
};
size_t matmul_workspace_bytes(int M, int N, int K, int b_rows);
hipError_t launch_matmul(const Matmul &a, bool bf16_out, hipStream_t stream);

// ---- gated linear recurrence (pf_gated.hip)
struct Gated {
    const void *X, *G, *Yin, *dY;      // Yin, dY: backward
    const float *h0, *dhL;
    void *Y, *dX, *dG;                 // Y: forward
    float *hL, *dh0;
    void *work;
    long long xb, xt, gb, gt, dyb, dyt;
    int B, L, D, gate, mix;
};
size_t gated_workspace_bytes(int B, int L, int D, bool is_bf16);
hipError_t launch_gated_fwd(const Gated &a, bool is_bf16, hipStream_t stream);
hipError_t launch_gated_bwd(const Gated &a, bool is_bf16, hipStream_t stream);

// ---- gated delta rule (pf_gdelta_flow.hip, pf_gdelta_scan.hip, pf_gdelta_grad.hip)
constexpr int kGDeltaChunk = 64, kGDeltaWidest = 256;
struct GDelta {
    const void *Q, *K, *V, *G, *beta, *dO;      // dO: backward
    long long qb, qt, qh, kb, kt, kh, vb, vt, vh, gb, gt, gh, bb, bt, bh, ob, ot, oh;      // strides: sequence, token, head
    const float *S0, *dSL;
    void *O, *dQ, *dK, *dV, *dG, *dbeta;
    float *SL, *dS0;
    const int *offsets;      // packed sequences: [N + 1]
    int N, L, Hk, Hv, dk, dv;      // L: tokens of every sequence, or rows of all packed ones together
    long long rows;          // rows of the outputs from one sequence to the next (packed: none)
    int per, chunks;         // chunks of a sequence (not of packed ones) and all together, or as many as there can be
    int *plan;               // the workspace's parts, set by gdelta_workspace
    __bf16 *T, *P, *Tt;      // Tt: backward
    float *vec, *S, *U, *Z, *R;
    float *ends, *starts, *fronts;      // of segments: states from zeros and of the unit matrix; states they start from; gradients from zeros
    int segments;            // of a sequence, run side by side (1: none are cut)
};
// d_k is padded with zeros to a width that the kernels have
__host__ __device__ inline int gdelta_width(int dk) { return dk <= 64 ? 64 : dk <= 128 ? 128 : 256; }
// values of one state in the workspace (the backward puts 64 rows of d_k in its place)
__host__ __device__ inline long long gdelta_state(const GDelta &a) { return (long long)gdelta_width(a.dk) * (a.dv <= 64 ? 64 : (a.dv + 31) / 32 * 32); }
// whether rows of Q and K are whole widths at multiples of 16 bytes
inline bool gdelta_full(const GDelta &a, int size)
{
    const uintptr_t all = reinterpret_cast<uintptr_t>(a.Q) | reinterpret_cast<uintptr_t>(a.K) | (uintptr_t)((a.qb | a.qt | a.qh | a.kb | a.kt | a.kh) * size);
    return a.dk == gdelta_width(a.dk) && all % 16 == 0;
}
// Segments that sequences are cut into, where their chains are few: each is run twice, the first time with as many rows more as the state has
// columns, and what joins them takes them one after the other.  Of that first run two workgroups to a compute unit at most, eight chunks to a
// segment at least, and no more segments than make a step of the join (1.7 us) worth the chunks (1.5 us, twice) that it saves; it pays from three
// segments and 32 chunks on.  bf16, heads of 128, forward, cut and whole: 65536 tokens of one head 215 and 1554 us, of four 586 and 1893, of eight
// 1122 and 2009; 2048 tokens of one head 49 and 63, 1600 in three segments 51 and 51 (their backward 138 and 121).  Backward: 16384 tokens of one head
// 250 and 881, of eight 866 and 1155, 2048 of one 125 and 147.  fp32: 65536 of one 366 and 3474, 2048 78 and 127, backward 196 and 263.  Heads of 64: 65536 of four
// 265 and 1367, 2048 of one 43 and 52, backward 98 and 122; of 256: 65536 of one 557 and 2587, 2048 91 and 98, backward 252 and 251 (nothing there).
inline int gdelta_segments(const GDelta &a)
{
    if (a.chunks == 0 || a.N == 0) return 1;
    const double chains = (double)a.N * a.Hv * ((a.dv + 31) / 32 * 32 + gdelta_width(a.dk)) / 16;
    const int chunks = a.chunks / a.N;
    int n = chains < 512 ? (int)(512 / chains) : 1;
    n = n < chunks / 8 ? n : chunks / 8;
    while (n > 1 && 2ll * n * n > 3ll * chunks) --n;
    return n < 3 || chunks < 32 ? 1 : n;
}
// Bytes of the workspace; a's parts of it, where `at` is not NULL.
size_t gdelta_workspace(GDelta &a, bool backward, void *at);
hipError_t launch_gdelta_fwd(const GDelta &a, bool is_bf16, hipStream_t stream);
hipError_t launch_gdelta_bwd(const GDelta &a, bool is_bf16, hipStream_t stream);
hipError_t launch_gdelta_flow(const GDelta &a, bool is_bf16, hipStream_t stream);
hipError_t launch_gdelta_scan(const GDelta &a, bool is_bf16, bool backward, hipStream_t stream);      // backward: leaves states and U
hipError_t launch_gdelta_scan_bwd(const GDelta &a, bool is_bf16, hipStream_t stream);
hipError_t launch_gdelta_grad(const GDelta &a, bool is_bf16, hipStream_t stream);

// ---- one token of the gated delta rule (pf_gdelta_step.hip)
struct GDeltaStep {
    const void *Q, *K, *V, *G, *beta;
    long long qb, qh, kb, kh, vb, vh, gb, gh, bb, bh;
    float *S;
    const int *slots;
    void *O;
    int B, pool, Hk, Hv, dk, dv;
};
hipError_t launch_gdelta_step(const GDeltaStep &a, bool is_bf16, hipStream_t stream);

// ---- norm and rotation of heads (pf_heads.hip)
constexpr int kHeadUnits = 64;      // lanes that a row can take
constexpr int kHeadsMost = 1 << 24; // heads of a token, queries and keys (counted in 32 bits)
inline int head_units(int d, int rot) { return (rot / 2 + 7) / 8 + (d - rot + 15) / 16; }
struct HeadSide {
    const void *X, *w, *dY;
    void *Y;                 // the output; of the backward: dX
    float *dw;
    long long xt, xh, dyt, dyh;      // strides: token, head
    int H;
    float scale;
};
struct Heads {
    HeadSide side[2];        // queries, keys
    const float *table;
    const int *positions;
    float *part;             // backward: sums for dw, [heads_bwd_parts][d]
    int M, d, rot, far, pairs, l2;
    float eps;
};
int heads_bwd_parts(int M, int Hq, int Hk, int d, int rot);
hipError_t launch_heads_fwd(const Heads &a, bool is_bf16, hipStream_t stream);
hipError_t launch_heads_bwd(const Heads &a, bool is_bf16, hipStream_t stream);

}  // namespace pf
