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

}  // namespace pf
