// Gated delta rule, backward: gradients of Q, K, beta and the gates, chunk by chunk (pf_gdelta.h), from the states S before and the
// gradients R behind each chunk, U, Z and P.  With X = dO U^T, Y = -Z U^T:
//
//   dQ = gamma dO S + (D X) K                      X on and below the diagonal, Y below it
//   dK = (D X)^T Q + W K + W^T K + delta U R - beta gamma Z S ,   W = beta D Y
//   dbeta_i = z_i.v_i - gamma_i z_i.S k_i + sum over j of Y_ij D_ij k_i.k_j
//   dg_t = sum over i >= t of e_i  +  <R, S'> ,   <R, S'> = gamma_64 <R, S> + sum of delta_j u_j.R k_j ,
//   e_i  = gamma_i do_i.S q_i - delta_i u_i.R k_i - beta_i gamma_i z_i.S k_i
//          + sum over j < i of (X P + Y A)_ij - sum over j > i of (X P + Y A)_ji .
#include "pf_gdelta.h"

namespace pf {
namespace gd {
namespace {

// A workgroup of four wavefronts for each chunk and value head; wavefront w has the tokens 16 w ..  First the pairs of tokens, W1 = D X and W,
// which stay in LDS; then 64 columns (of d_k) of the gradients at a time, with 32 rows (of d_v) of S and R in LDS.  Where heads
// share Q and K, their parts of dQ and dK take the place of S and R in the workspace, and share_kernel adds them.
template <typename T, bool FULL>
__global__ __launch_bounds__(256) void grad_kernel(GDelta a)
{
    constexpr int ROWS = 32, COLS = 64, NC = COLS / 16, KP = pitch<T>(COLS);
    typedef Tile<T, 2, ROWS, COLS> StateTile;      // [d_v][d_k]
    typedef Tile<T, 2, C, ROWS> UTile;             // [token][d_v]
    typedef Tile<T, 2, C, C> PairTile;             // [j][i]
    constexpr int kStates = 2 * StateTile::kBytes, kTokens = C * KP * (int)sizeof(T);
    static_assert(UTile::kBytes <= kStates, "U comes in the place of S and R");
    __shared__ __attribute__((aligned(16))) char smem[kStates + 2 * kTokens + 2 * PairTile::kBytes];
    __shared__ float coarse[C], fine[C];
    __shared__ float srow[C], scol[4][C], sdot[4];
    const StateTile Ss = {reinterpret_cast<T *>(smem)}, Rs = {reinterpret_cast<T *>(smem + StateTile::kBytes)};
    const UTile Us = {reinterpret_cast<T *>(smem)};
    T *Ks = reinterpret_cast<T *>(smem + kStates), *Qs = reinterpret_cast<T *>(smem + kStates + kTokens);
    const PairTile W1 = {reinterpret_cast<T *>(smem + kStates + 2 * kTokens)}, W2 = {reinterpret_cast<T *>(smem + kStates + 2 * kTokens + PairTile::kBytes)};

    const int id = (int)xcd_consecutive(blockIdx.x, gridDim.x), chunk = id / a.Hv, h = id - chunk * a.Hv, share = a.Hv / a.Hk, hk = h / share;
    Chunk x;
    if (!chunk_at(a, chunk, x)) return;
    const int w = wave_id(), lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
    const int wide = (a.dv + 31) / 32 * 32, DK = gdelta_width(a.dk);
    const int mine = min(16 * w + r16, x.len - 1);      // this lane's row of the left operands
    const int i0 = 16 * w + 4 * g;                      // and its first row of the results

    const long long xi = (long long)chunk * a.Hv + h;
    const T *K = static_cast<const T *>(a.K) + x.seq * a.kb + x.tok * a.kt + hk * a.kh;
    const T *Q = static_cast<const T *>(a.Q) + x.seq * a.qb + x.tok * a.qt + hk * a.qh;
    const T *V = static_cast<const T *>(a.V) + x.seq * a.vb + (x.tok + mine) * a.vt + h * a.vh;
    const T *dO = static_cast<const T *>(a.dO) + x.seq * a.ob + (x.tok + mine) * a.ot + h * a.oh;
    const Vec vec = vec_at(a.vec, xi);
    float *S = a.S + xi * gdelta_state(a), *R = a.R + xi * gdelta_state(a);
    const float *U = a.U + xi * C * wide, *Z = a.Z + (xi * C + 16 * w + r16) * wide;
    // eight values of d_v of the lane's token: rows behind the end count as zeros
    auto o_at = [&](int v) { return fetch<T, false>(dO + v, 16 * w + r16 < x.len ? a.dv - v : 0); };

    if (threadIdx.x < C) coarse[threadIdx.x] = vec.coarse[threadIdx.x], fine[threadIdx.x] = vec.fine[threadIdx.x];
    const f32x4 gamma = *reinterpret_cast<const f32x4 *>(vec.gamma + i0), delta = *reinterpret_cast<const f32x4 *>(vec.delta + i0);
    const f32x4 beta = *reinterpret_cast<const f32x4 *>(vec.beta + i0);

    // ---- pairs of tokens; K K^T again, for Y A and its share of dbeta
    f32x4 X[4], Y[4], kk[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) X[n] = Y[n] = kk[n] = zero4();
    float zv = 0.f;
    struct {
        In<T> o, v;
        f32x8 z;
        f32x4 u[C * ROWS / 4 / 256];
    } next;      // the next step's loads, asked for a step ahead
    auto ask = [&](int v0) {
        next.o = o_at(v0 + 8 * g), next.v = fetch<T, false>(V + v0 + 8 * g, a.dv - v0 - 8 * g);
        next.z = *reinterpret_cast<const f32x8 *>(Z + v0 + 8 * g);
#pragma unroll
        for (int i = 0; i < C * ROWS / 4 / 256; ++i) {
            const int at = i * 256 + threadIdx.x;
            next.u[i] = *reinterpret_cast<const f32x4 *>(U + at / (ROWS / 4) * wide + v0 + 4 * (at % (ROWS / 4)));
        }
    };
    ask(0);
    for (int v0 = 0; v0 < wide; v0 += ROWS) {
        const In<T> of_o = next.o;
        const f32x8 z = next.z, v = in_f32(next.v);
#pragma unroll
        for (int e = 0; e < 8; ++e) zv += z[e] * v[e];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < C * ROWS / 4 / 256; ++i) {
            const int at = i * 256 + threadIdx.x;
            Us.put4(at / (ROWS / 4), 4 * (at % (ROWS / 4)), next.u[i]);
        }
        ask(min(v0 + ROWS, wide - ROWS));
        __syncthreads();
        const Of<T, 2> of_z = of<T, 2>(z);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const Of<T, 2> u = Us.rows(16 * n + r16, 8 * g);
            X[n] = mma<2>(of_o, u, X[n]);
            Y[n] = mma22<T>(of_z, u, Y[n]);
        }
    }
    zv = sum_of_groups(zv);      // of token 16 w + r16
    In<T> kn[5];
    auto keys = [&](int k) {
        kn[4] = fetch<T, FULL>(K + mine * a.kt + k, a.dk - k);
#pragma unroll
        for (int n = 0; n < 4; ++n) kn[n] = fetch<T, FULL>(K + min(16 * n + r16, x.len - 1) * a.kt + k, a.dk - k);
    };
    keys(8 * g);
    for (int k = 8 * g; k < DK; k += 32) {
        In<T> now[5];
#pragma unroll
        for (int n = 0; n < 5; ++n) now[n] = kn[n];
        keys(min(k + 32, DK - 32 + 8 * g));
#pragma unroll
        for (int n = 0; n < 4; ++n) kk[n] = mma(now[4], now[n], kk[n]);
    }
    const bf16 *Pt = a.P + xi * kMatrix;      // of the transpose, in three parts
    f32x4 row = zero4(), yk = zero4();
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int j = 16 * n + r16;
        f32x4 w1 = zero4(), w2 = zero4();
        float col = 0.f;
        if (n <= w) {
            const float cj = coarse[j], fj = fine[j];
            f32x4 p = zero4();
#pragma unroll
            for (int q = 2; q >= 0; --q)
                p += __builtin_convertvector(ld4(Pt + ((high_fragment(n, w >> 1) * 3 + q) * 64 + r16 + 16 * (2 * (w & 1) + (g >> 1))) * 8 + 4 * (g & 1)), f32x4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = i0 + e;
                const float D = power(coarse[i] - cj, fine[i] - fj);
                const bool in = i < x.len;
                w1[e] = in && j <= i ? D * X[n][e] : 0.f;
                const float y = in && j < i ? -Y[n][e] * D : 0.f;
                w2[e] = beta[e] * y;
                yk[e] += y * kk[n][e];
                const float both = (in && j < i ? X[n][e] * p[e] : 0.f) + w2[e] * kk[n][e];
                row[e] += both;
                col += both;
            }
        }
        W1.put4(j, i0, w1);
        W2.put4(j, i0, w2);
        col = sum_of_groups(col);
        if (g == 0) scol[w][j] = col;
    }

    // ---- 64 columns of dQ and dK at a time
    f32x4 oq = zero4(), uk = zero4(), zk = zero4();
    float dot = 0.f;
    constexpr int NS = ROWS * COLS / 4 / 256, NK = C * COLS / 8 / 256;
    struct {
        In<T> o;
        f32x8 u, z;
        f32x4 s[NS], r[NS];
    } step;      // the next step's, and the next columns of K and Q
    In<T> kr[NK], qr[NK];
    auto states = [&](int c0, int v0) {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int at = i * 256 + threadIdx.x, from = (v0 + at / (COLS / 4)) * DK + c0 + 4 * (at % (COLS / 4));
            step.s[i] = *reinterpret_cast<const f32x4 *>(S + from), step.r[i] = *reinterpret_cast<const f32x4 *>(R + from);
        }
        step.o = o_at(v0 + 8 * g);
        step.u = *reinterpret_cast<const f32x8 *>(U + (16 * w + r16) * wide + v0 + 8 * g);
        step.z = *reinterpret_cast<const f32x8 *>(Z + v0 + 8 * g);
    };
    auto columns = [&](int c0) {
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int at = i * 256 + threadIdx.x, from = min(at / (COLS / 8), x.len - 1), k = c0 + 8 * (at % (COLS / 8));
            kr[i] = fetch<T, FULL>(K + from * a.kt + k, a.dk - k), qr[i] = fetch<T, FULL>(Q + from * a.qt + k, a.dk - k);
        }
    };
    columns(0);
    states(0, 0);
    for (int c0 = 0; c0 < DK; c0 += COLS) {
        f32x4 oS[NC], uR[NC], zS[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) oS[n] = uR[n] = zS[n] = zero4();
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int at = i * 256 + threadIdx.x, to = at / (COLS / 8) * KP + 8 * (at % (COLS / 8));
            __builtin_memcpy(__builtin_assume_aligned(Ks + to, 16), &kr[i], sizeof(kr[i]));
            __builtin_memcpy(__builtin_assume_aligned(Qs + to, 16), &qr[i], sizeof(qr[i]));
        }
        const int behind = min(c0 + COLS, DK - COLS);
        columns(behind);
        for (int v0 = 0; v0 < wide; v0 += ROWS) {
            const In<T> of_o = step.o;
            const f32x8 u = step.u, z = step.z;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const int at = i * 256 + threadIdx.x, r = at / (COLS / 4), k = 4 * (at % (COLS / 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) dot += step.s[i][e] * step.r[i][e];
                Ss.put4(r, k, step.s[i]);
                Rs.put4(r, k, step.r[i]);
            }
            const bool over = v0 + ROWS >= wide;
            states(over ? behind : c0, over ? 0 : v0 + ROWS);
            __syncthreads();
            const Of<T, 2> of_z = of<T, 2>(z), of_u = of<T, 2>(u);
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const Of<T, 2> sf = Ss.cols(8 * g, 16 * n, r16), rf = Rs.cols(8 * g, 16 * n, r16);
                oS[n] = mma<2>(of_o, sf, oS[n]);
                zS[n] = mma22<T>(of_z, sf, zS[n]);
                uR[n] = mma22<T>(of_u, rf, uR[n]);
            }
        }
        // what a row of these products and a row of Q or K have in common; dQ and dK so far
        f32x4 dq[NC], dk[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float k = to_f32(Ks[(i0 + e) * KP + 16 * n + r16]), q = to_f32(Qs[(i0 + e) * KP + 16 * n + r16]);
                oq[e] += oS[n][e] * q;
                uk[e] += uR[n][e] * k;
                zk[e] += zS[n][e] * k;
            }
            dq[n] = gamma * oS[n];
            dk[n] = delta * uR[n] - beta * gamma * zS[n];
            __builtin_amdgcn_sched_barrier(0);      // (values of one tile at a time in registers)
        }
        // dQ += W1 K, dK += W1^T Q + W2 K + W2^T K, tokens in steps of 32 (what the triangles leave out is zeros)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            LDS_FENCE();
            const int k0 = 32 * t + 8 * g;
            const bool low = t <= w / 2, high = t >= w / 2;
            Of<T, 2> w1, wl, w1t, wu;
            if (low) w1 = W1.cols(k0, 16 * w, r16), wl = W2.cols(k0, 16 * w, r16);
            if (high) w1t = W1.rows(16 * w + r16, k0), wu = W2.rows(16 * w + r16, k0);
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const In<T> k = frag_cols(Ks, KP, k0, 16 * n, r16);
                if (low) dq[n] = mma<2>(w1, k, dq[n]), dk[n] = mma<2>(wl, k, dk[n]);
                if (high) dk[n] = mma<2>(wu, k, dk[n]), dk[n] = mma<2>(w1t, frag_cols(Qs, KP, k0, 16 * n, r16), dk[n]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (share > 1) {      // (these columns of S and R have been read, and no others are written)
            __syncthreads();
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int to = (i0 + e) * DK + c0 + 16 * n + r16;
                    S[to] = dq[n][e];
                    R[to] = dk[n][e];
                }
        } else {
            const long long at = (out_row(a, x.seq, x.tok + i0) * a.Hk + hk) * a.dk + c0 + r16, step = (long long)a.Hk * a.dk;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (i0 + e >= x.len) continue;
                T *q = static_cast<T *>(a.dQ) + at + e * step, *k = static_cast<T *>(a.dK) + at + e * step;
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    if (c0 + 16 * n + r16 < a.dk) q[16 * n] = (T)dq[n][e], k[16 * n] = (T)dk[n][e];
            }
        }
    }

    // ---- beta and the gates
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        oq[e] = gamma[e] * sum_of_16(oq[e]), uk[e] = delta[e] * sum_of_16(uk[e]), zk[e] = gamma[e] * sum_of_16(zk[e]);
        row[e] = sum_of_16(row[e]), yk[e] = sum_of_16(yk[e]);
        const int i = i0 + e;
        const float zvi = __shfl(zv, 4 * g + e);
        if (r16 == 0) {
            srow[i] = oq[e] - uk[e] - beta[e] * zk[e] + row[e];
            if (i < x.len) static_cast<T *>(a.dbeta)[out_row(a, x.seq, x.tok + i) * a.Hv + h] = (T)(zvi - zk[e] + yk[e]);
        }
    }
    {      // <R, S'>: every wavefront's part of gamma_64 <R, S>, and of its tokens' delta u.R k (none behind the end, where u = 0)
        const float sum = sum_of_groups(uk[0] + uk[1] + uk[2] + uk[3]);
        dot = sum_of_groups(sum_of_16(dot));
        if (lane == 0) sdot[w] = vec.gamma[C - 1] * dot + sum;
    }
    __syncthreads();
    if (w == 0) {      // sums from the chunk's end
        float e = lane < x.len ? srow[lane] - (scol[0][lane] + scol[1][lane] + scol[2][lane] + scol[3][lane]) : 0.f;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const float other = __shfl_down(e, s);
            if (lane + s < 64) e += other;
        }
        e += sdot[0] + sdot[1] + sdot[2] + sdot[3];
        if (lane < x.len) static_cast<T *>(a.dG)[out_row(a, x.seq, x.tok + lane) * a.Hv + h] = (T)e;
    }
}

// dQ and dK of a chunk and a head of keys out of the parts of the value heads that share it, in their order.
template <typename T> __global__ __launch_bounds__(256) void share_kernel(GDelta a)
{
    const int chunk = blockIdx.x / a.Hk, hk = blockIdx.x - chunk * a.Hk, share = a.Hv / a.Hk, DK = gdelta_width(a.dk);
    Chunk x;
    if (!chunk_at(a, chunk, x)) return;
    const long long each = gdelta_state(a), first = ((long long)chunk * a.Hv + hk * share) * each;
    for (int u = threadIdx.x; u < x.len * DK / 4; u += 256) {
        const int i = 4 * u / DK, c = 4 * u - i * DK;
        if (c >= a.dk) continue;
        f32x4 q = zero4(), k = zero4();
        for (int s = 0; s < share; ++s) {
            q += *reinterpret_cast<const f32x4 *>(a.S + first + s * each + 4 * u);
            k += *reinterpret_cast<const f32x4 *>(a.R + first + s * each + 4 * u);
        }
        const long long at = (out_row(a, x.seq, x.tok + i) * a.Hk + hk) * a.dk + c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < a.dk) static_cast<T *>(a.dQ)[at + e] = (T)q[e], static_cast<T *>(a.dK)[at + e] = (T)k[e];
    }
}

template <typename T> hipError_t grad(const GDelta &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((long long)a.chunks * a.Hv));
    gdelta_full(a, sizeof(T)) ? grad_kernel<T, true><<<grid, 256, 0, stream>>>(a) : grad_kernel<T, false><<<grid, 256, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.Hv == a.Hk) return hipSuccess;
    share_kernel<T><<<dim3((unsigned)((long long)a.chunks * a.Hk)), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace
}  // namespace gd

hipError_t launch_gdelta_grad(const GDelta &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? gd::grad<bf16>(a, stream) : gd::grad<float>(a, stream);
}

}  // namespace pf
