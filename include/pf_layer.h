/*
 * pf_layer.h - C ABI of the operators of a layer around the delta rule of pf.h, MI355X (gfx950): the norm in front of
 *              its projections, the projections in 8 bits, and the gated linear recurrence, which is the flow of
 *              Section 3.1 of ParallelFlow (arXiv 2504.00492) with diagonal drivers.  Forward and backward.
 *              Library: libpf_layer.so (it loads libpf.so for pf_status_str and pf_version).
 *
 * Conventions: those of pf.h.  Every data pointer is a DEVICE pointer owned by the caller, base addresses are 16-byte
 * aligned (PF_ERR_ALIGN; of inputs that come with strides: aligned to their elements), the library never allocates, frees or synchronises, work is enqueued on `stream`, every
 * argument check happens on the host before anything is launched, errors are return codes.  Calls that share a workspace
 * or outputs must be ordered by the caller.  Results do not depend on timing: the same call on the same device gives the
 * same bits.  A row or sequence in a call of other sizes may take another kernel, or sums in another order, and differ in its last
 * bits.  Sums, statistics and states are held in fp32.  In addition
 *   - the innermost dimension of every array is contiguous; where a row stride (ld...) is an argument, it is in elements, at
 *     least the row's length (PF_ERR_SHAPE) and otherwise free; batch and token strides are not negative and otherwise free;
 *   - outputs must not overlap inputs, except where an entry says so;
 *   - "8 bits" is the e4m3 format without infinities (largest value 448; conversions round to nearest even), always with
 *     fp32 scales that the stored value is multiplied by.  The arrays of scales are stored block by block:
 *     scale[b][row] belongs to columns 128 b .. 128 b + 127 of `row` (the last block may be shorter);
 *   - NaN and infinities in inputs reach the outputs that depend on them.
 */
#ifndef PF_LAYER_H
#define PF_LAYER_H

#include "pf.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Of every call here: a size that needs more workgroups than one launch holds (2^32 threads) is PF_ERR_UNSUPPORTED. */

/*
 * Root-mean-square norm of rows, with the residual's addition before it and an output in 8 bits.
 *
 *   s = round(x + r)                         (s = x without R)
 *   y = s / sqrt(mean(s^2) + eps) * w        (mean over the row)
 *
 *   X      [M, D], row stride ldx   dt    in
 *   R      [M, D], row stride ldr   dt    in    the residual stream; NULL: none
 *   w      [D]                      dt    in    NULL: ones
 *   S      [M, D]                   dt    out   NULL: not written.  S == X or S == R is allowed where that is dense
 *   Y      [M, D]                   dt    out   NULL: not written
 *   Q      [M, D], row stride ldq   e4m3  out   y in 8 bits, a scale for each row and block of 128 columns; NULL: not
 *                                               written.  ldq: a multiple of 16; the bytes behind a row's D stay
 *   scale  [ceil(D/128), M]         fp32  out   with Q
 *
 * With m = max(max|y| over the block, 1e-30): scale = m / 448, Q = e4m3(y * 448 / m).  At least one of Y and Q is
 * wanted (PF_ERR_NULL).  D up to 16384 (pf_norm_supported; else PF_ERR_UNSUPPORTED).  M == 0: nothing is done, and the
 * pointers may be NULL.  A row of zeros with eps = 0 gives NaN.  Squares are summed in fp32: where their sum overflows (values of
 * 1e19), y is zero.
 */
int pf_norm_supported(int D, pf_dtype dt);
pf_status pf_norm_fwd(const void *X, long long ldx, const void *R, long long ldr, const void *w, void *S, void *Y,
                      void *Q, long long ldq, float *scale, int M, int D, float eps, pf_dtype dt, pf_stream stream);

/*
 * Its backward.  With xh = s / sqrt(mean(s^2) + eps), g = w dy (a rounding to 8 bits passes its gradient on unchanged):
 *
 *   dx = ds + (g - xh mean(g xh)) / sqrt(mean(s^2) + eps)       (the gradient of x and of r alike)
 *   dw = sum over rows of dy xh
 *
 *   S      [M, D], row stride lds    dt    in    the stored sum (x itself without a residual)
 *   w      [D]                       dt    in    NULL: ones
 *   dY     [M, D], row stride lddy   dt    in
 *   dS     [M, D], row stride ldds   dt    in    gradient that reaches s past the norm; NULL: none
 *   dX     [M, D]                    dt    out   dX == dS or dX == dY is allowed where that is dense
 *   dw     [D]                       fp32  out   NULL: not wanted (then no workspace either).  M == 0: zeros
 *   workspace / workspace_bytes            at least pf_norm_bwd_workspace_bytes(...) bytes, overwritten
 */
size_t pf_norm_bwd_workspace_bytes(int M, int D);
pf_status pf_norm_bwd(const void *S, long long lds, const void *w, const void *dY, long long lddy, const void *dS,
                      long long ldds, void *dX, float *dw, int M, int D, float eps, pf_dtype dt, void *workspace,
                      size_t workspace_bytes, pf_stream stream);

/*
 * A matrix in 8 bits.  rows = 1: a scale for each row and 128 columns; rows = 128: one for each square of 128 x 128
 * (weights).  Also, or instead, the transposed matrix, whose blocks run along ITS rows (128 rows of X by one column, or
 * the same squares): the operand of a product that sums over the rows of X.
 *
 *   X       [M, K], row stride ldx     dt    in
 *   Q       [M, K], row stride ldq     e4m3  out   NULL: not wanted
 *   scale   [ceil(K/128), M] or [ceil(K/128), ceil(M/128)]   fp32   out   with Q
 *   QT      [K, M], row stride ldqt    e4m3  out   NULL: not wanted
 *   scaleT  [ceil(M/128), K] or [ceil(M/128), ceil(K/128)]   fp32   out   with QT
 *
 * With m = max(max|x| over the block, 1e-30): scale = m * (1/448), Q = e4m3(x * (1/m * 448)), each operation in fp32.
 * ldq, ldqt: multiples of 16; the bytes behind a row stay.  At least one of Q and QT (PF_ERR_NULL).  M == 0 or K == 0:
 * nothing is done.
 */
pf_status pf_quant_fp8(const void *X, long long ldx, void *Q, long long ldq, float *scale, void *QT, long long ldqt,
                       float *scaleT, int M, int K, int rows, pf_dtype dt, pf_stream stream);

/*
 * Product of two matrices in 8 bits, the second transposed:
 *
 *   C[m, n] = sum over blocks b of  sa[b, m] sb[b, n / b_rows]  sum over k in b of  A[m, k] B[n, k]
 *
 *   A   [M, K], row stride lda     e4m3   in    lda, ldb: multiples of 16, and every row, the last one too, lies in whole 16
 *                                               bytes (what these hold behind a row's K is not used)
 *   sa  [ceil(K/128), M]           fp32   in
 *   B   [N, K], row stride ldb     e4m3   in    weights [out, in] for a forward; b_rows = 128: squares of 128 x 128
 *   sb  [ceil(K/128), N] (b_rows = 1) or [ceil(K/128), ceil(N/128)] (b_rows = 128)   fp32   in
 *   C   [M, N], row stride ldc     dt     out
 *   workspace / workspace_bytes           at least pf_matmul_fp8_workspace_bytes(...) bytes, overwritten (may be NULL
 *                                         when that is 0, as for M up to 16)
 *
 * dt = PF_BF16: the sum over a block is the 8-bit matrix instruction's, which adds eight neighbouring products at a time aligned to
 * the largest of them and drops what lies 2^-13 below that: 7 * 2^-13 of the largest of every eight at most, 1.4e-5 of the result's norm
 * for normally distributed values; it shows where loud columns cancel.  A caller to whom that matters takes PF_F32 and rounds.
 * dt = PF_F32: exact products, fp32 sums.  Blocks are joined by one fp32 fma each, with sa sb, rounded to fp32, as the factor.  The gradient of A's
 * source is the same product on dY and the transposed copy of B, that of B's on the transposed copies of dY and A's source
 * (pf_quant_fp8).  b_rows other than 1 and 128: PF_ERR_UNSUPPORTED.  M == 0 or N == 0: nothing is done; K from 1 to
 * 2^31 - 128 (PF_ERR_UNSUPPORTED beyond).
 */
size_t pf_matmul_fp8_workspace_bytes(int M, int N, int K, int b_rows);
pf_status pf_matmul_fp8(const void *A, long long lda, const float *sa, const void *B, long long ldb, const float *sb,
                        int b_rows, void *C, long long ldc, int M, int N, int K, pf_dtype dt, void *workspace,
                        size_t workspace_bytes, pf_stream stream);

/*
 * Gated linear recurrence: per sequence and channel, from h_0 = h0,
 *
 *   h_t = a_t h_{t-1} + b_t ,   y_t = round(h_t)            t = 1 .. L
 *
 *   gate = PF_GATE_VALUE   a = g (any value)     mix = 0   b = x
 *          PF_GATE_LOG     a = exp(g)            mix = 1   b = (1 - a) x
 *          PF_GATE_LOGIT   a = 1 / (1 + exp(-g))
 *
 * a = 0 (a log of minus infinity) starts a sequence anew: packed sequences need nothing else.  The recurrence runs on the
 * unrounded h.
 *
 *   X   [B, L, D], strides xb (batch), xt (token)   dt     in
 *   G   [B, L, D], strides gb, gt                   dt     in
 *   h0  [B, D]                                      fp32   in    NULL: zeros
 *   Y   [B, L, D]                                   dt     out
 *   hL  [B, D]                                      fp32   out   NULL: not written.  hL == h0 is allowed
 *   workspace / workspace_bytes                     at least pf_gated_workspace_bytes(...) bytes, overwritten (may be
 *                                                   NULL when that is 0, as for L up to 16; the forward and the
 *                                                   backward need the same)
 *
 * L == 0: hL receives h0 (or zeros), the sequence pointers may be NULL.  B == 0: nothing is done.  L up to 2^30
 * (PF_ERR_UNSUPPORTED).
 * Where the same recurrence over the sizes |a|, |b|, |h0| stays inside fp32, this one does too, however far products of gates leave it;
 * where that one overflows, values may be infinite or NaN from there on.
 */
typedef enum { PF_GATE_VALUE = 0, PF_GATE_LOG = 1, PF_GATE_LOGIT = 2 } pf_gate;

size_t pf_gated_workspace_bytes(int B, int L, int D, pf_dtype dt);
pf_status pf_gated_fwd(const void *X, long long xb, long long xt, const void *G, long long gb, long long gt,
                       const float *h0, void *Y, float *hL, int B, int L, int D, pf_gate gate, int mix, pf_dtype dt,
                       void *workspace, size_t workspace_bytes, pf_stream stream);

/*
 * Its backward, from the stored y.  From l_{L+1} = 0, with dy_L counting dhL in:
 *
 *   l_t = dy_t + a_{t+1} l_{t+1} ,   db_t = l_t ,   da_t = l_t y_{t-1} ,   dh0 = a_1 l_1          (y_0 = h0)
 *   dx = db, or (1 - a) db with the mix, which also takes l_t x_t off da_t;
 *   dg = da, a da or a (1 - a) da by the gate's form
 *
 *   X, G, h0           as above (X is not read without the mix and may be NULL then)
 *   Y   [B, L, D]                                     dt     in
 *   dY  [B, L, D], strides dyb, dyt                   dt     in
 *   dhL [B, D]                                        fp32   in    NULL: zeros
 *   dX, dG [B, L, D]                                  dt     out
 *   dh0 [B, D]                                        fp32   out   NULL: not written.  dh0 == dhL is allowed
 */
pf_status pf_gated_bwd(const void *X, long long xb, long long xt, const void *G, long long gb, long long gt,
                       const float *h0, const void *Y, const void *dY, long long dyb, long long dyt, const float *dhL,
                       void *dX, void *dG, float *dh0, int B, int L, int D, pf_gate gate, int mix, pf_dtype dt,
                       void *workspace, size_t workspace_bytes, pf_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* PF_LAYER_H */
