// Gated delta rule, backward: gradients of Q, K, beta and the gates, chunk by chunk (pf_gdelta.h), from the states S before and the
// gradients R behind each chunk, U, Z and P.  With X = dO U^T, Y = -Z U^T:
//
//   dQ = gamma dO S + (D X) K                      X on and below the diagonal, Y below it
//   dK = (D X)^T Q + W K + W^T K + delta U R - beta gamma Z S ,   W = beta D Y
//   dbeta_i = z_i.u_i / beta_i ,  and where beta_i is 0  z_i.v_i - gamma_i z_i.S k_i + sum over j of Y_ij D_ij k_i.k_j
//   dg_t = sum over i >= t > j of M_ij + sum over i >= t of (gamma_i do_i.S q_i - beta_i gamma_i z_i.S k_i)
//          + sum over j < t of delta_j u_j.R k_j + gamma_64 <R, S> ,   M = X P + Y A .
//
// Every term of dg_t is of what goes from tokens before t, or the state, to t and later ones, or the next state, so it has t's gate in it.  (As
// differences of sums over whole rows and columns of M the same cost 2e-5 of the gradient at gates of -5, all of it at -16.)
#include "pf_gdelta.h"

namespace pf {
namespace gd {
namespace {

template <typename T> __device__ __forceinline__ In<T> kept(In<T> x, bool keep)
{
    uint32_t w[sizeof(x) / 4];
    __builtin_memcpy(w, &x, sizeof(x));
#pragma unroll
    for (uint32_t &v : w) v = keep ? v : 0;
    __builtin_memcpy(&x, w, sizeof(x));
    return x;
}

// FULL: rows of Q, K, V and dO are whole widths at multiples of 16 bytes.
// A workgroup of eight wavefronts for each chunk and value head; wavefronts w and w + 4 have the tokens 16 w .., of each result one half of the
// columns.  COLS columns (of d_k) of the gradients at a time, so all of them up to 128: with 32 rows (of d_v) of S, R and U in LDS the products with
// them, the first time X and Y too, so that each is read once; then W1 = D X and W, which stay in LDS, and the products with K and Q.
// What bounds it is memory, 310 KB a workgroup at 128 x 128 in bf16: 4096 of them take 392 us, 3.3 TB/s (with 64 columns at a time, U and Z
// read three times, 575; of four wavefronts and no load ahead 640).  One workgroup to a compute unit, by its registers and by its LDS
// (119 KB of 160 in bf16, 87 with 64 columns), though not all of that is in use at any one time.
// Where heads share Q and K, their parts of dQ and dK take the place of S and R in the workspace, and share_kernel adds them.
template <typename T, int COLS, bool FULL>
__global__ __launch_bounds__(512) void grad_kernel(GDelta a)
{
    constexpr int ROWS = 32, NC = COLS / 32, NP = C / 32, KP = pitch<T>(COLS), THREADS = 512;
    typedef Tile<T, 2, ROWS, COLS> StateTile;      // [d_v][d_k]
    typedef Tile<T, 2, C, ROWS> UTile;             // [token][d_v]
    typedef Tile<T, 2, C, C> PairTile;             // [j][i]
    constexpr int kTokens = C * KP * (int)sizeof(T);
    __shared__ __attribute__((aligned(16))) char states[2][StateTile::kBytes], values[UTile::kBytes], tokens[2][kTokens], pairs[2][PairTile::kBytes];
    __shared__ __attribute__((aligned(16))) float rows[3][C];      // gamma, delta, beta
    __shared__ float coarse[C], fine[C];
    __shared__ float srow[2][C], sstate[2][C], slater[2][C], sbeta[2][C], szu[C], scol[4][C], sdot[8];
    const StateTile Ss = {reinterpret_cast<T *>(states[0])}, Rs = {reinterpret_cast<T *>(states[1])};
    const UTile Us = {reinterpret_cast<T *>(values)};
    T *Ks = reinterpret_cast<T *>(tokens[0]), *Qs = reinterpret_cast<T *>(tokens[1]);
    const PairTile W1 = {reinterpret_cast<T *>(pairs[0])}, W2 = {reinterpret_cast<T *>(pairs[1])};

    const int id = (int)xcd_consecutive(blockIdx.x, gridDim.x), chunk = id / a.Hv, h = id - chunk * a.Hv, share = a.Hv / a.Hk, hk = h / share;
    Chunk x;
    if (!chunk_at(a, chunk, x)) return;
    const int w = wave_id() & 3, half = wave_id() >> 2;
    int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
    auto again = [&] {      // addresses from here on are worked out here: held over a pass, they take the registers of the products
        asm volatile("" : "+v"(lane));
        r16 = lane & 15, g = lane >> 4;
    };
    const int wide = (a.dv + 31) / 32 * 32, DK = gdelta_width(a.dk);
    const int mine = min(16 * w + r16, x.len - 1);      // this lane's row of the left operands

    const long long xi = (long long)chunk * a.Hv + h;
    const T *K = static_cast<const T *>(a.K) + x.seq * a.kb + x.tok * a.kt + hk * a.kh;
    const T *Q = static_cast<const T *>(a.Q) + x.seq * a.qb + x.tok * a.qt + hk * a.qh;
    const T *V = static_cast<const T *>(a.V) + x.seq * a.vb + (x.tok + mine) * a.vt + h * a.vh;
    const T *dO = static_cast<const T *>(a.dO) + x.seq * a.ob + (x.tok + mine) * a.ot + h * a.oh;
    const Vec vec = vec_at(a.vec, xi);
    float *S = a.S + xi * gdelta_state(a), *R = a.R + xi * gdelta_state(a);
    const float *U = a.U + xi * C * wide, *Z = a.Z + (xi * C + 16 * w + r16) * wide;
    const bf16 *Pt = a.P + xi * kMatrix;      // of the transpose, in three parts

    // a step's loads are asked for a step ahead
    constexpr int NS = ROWS * COLS / 4 / THREADS, NK = C * COLS / 8 / THREADS;
    const int urow = threadIdx.x / (ROWS / 4), ucol = 4 * (threadIdx.x % (ROWS / 4));
    const bool here = 16 * w + r16 < x.len;      // (rows of dO behind the end count as zeros)
    struct {
        In<T> o, v;
        f32x8 z;
        f32x4 u, s[NS], r[NS];
    } next;
    auto ask = [&](int c0, int v0) {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int at = i * THREADS + threadIdx.x, from = (v0 + at / (COLS / 4)) * DK + c0 + 4 * (at % (COLS / 4));
            next.s[i] = *reinterpret_cast<const f32x4 *>(S + from), next.r[i] = *reinterpret_cast<const f32x4 *>(R + from);
        }
        next.u = *reinterpret_cast<const f32x4 *>(U + urow * wide + v0 + ucol);
        next.z = *reinterpret_cast<const f32x8 *>(Z + v0 + 8 * g);
        if constexpr (FULL) {
            next.o = kept(fetch<T, true>(dO + v0 + 8 * g, 8), here);      // (a branch around the load would wait for it)
            next.v = fetch<T, true>(V + v0 + 8 * g, 8);
        } else {
            next.o = fetch<T, false>(dO + v0 + 8 * g, here ? a.dv - v0 - 8 * g : 0);
        }
    };
    if (threadIdx.x < C) coarse[threadIdx.x] = vec.coarse[threadIdx.x], fine[threadIdx.x] = vec.fine[threadIdx.x];
    else if (threadIdx.x < 4 * C) (&rows[0][0])[threadIdx.x - C] = (threadIdx.x < 2 * C ? vec.gamma : threadIdx.x < 3 * C ? vec.delta : vec.beta)[threadIdx.x % C];

    auto ld_rows = [&](int i) { return *reinterpret_cast<const f32x4 *>(rows[i] + 16 * w + 4 * g); };      // (of the results' rows)
    f32x4 X[NP], Y[NP];      // of the tokens 16 (2 m + half) ..
#pragma unroll
    for (int m = 0; m < NP; ++m) X[m] = Y[m] = zero4();
    f32x4 row = zero4(), yk = zero4(), oq = zero4(), uk = zero4(), zk = zero4();
    float zv = 0.f, dot = 0.f;
    const int nh = 16 * NC * half;      // this wavefront's columns
    for (int c0 = 0; c0 < DK; c0 += COLS) {
        ask(c0, 0);
        In<T> kr[NK], qr[NK];
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int at = i * THREADS + threadIdx.x, from = min(at / (COLS / 8), x.len - 1), k = c0 + 8 * (at % (COLS / 8));
            kr[i] = fetch<T, FULL>(K + from * a.kt + k, a.dk - k), qr[i] = fetch<T, FULL>(Q + from * a.qt + k, a.dk - k);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int at = i * THREADS + threadIdx.x, to = at / (COLS / 8) * KP + 8 * (at % (COLS / 8));
            __builtin_memcpy(__builtin_assume_aligned(Ks + to, 16), &kr[i], sizeof(kr[i]));
            __builtin_memcpy(__builtin_assume_aligned(Qs + to, 16), &qr[i], sizeof(qr[i]));
        }
        f32x4 oS[NC], uR[NC], zS[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) oS[n] = uR[n] = zS[n] = zero4();
        for (int v0 = 0; v0 < wide; v0 += ROWS) {
            __syncthreads();
            const In<T> of_o = next.o;
            const f32x8 z = next.z;
            if (c0 == 0) {
                if constexpr (!FULL) next.v = fetch<T, false>(V + v0 + 8 * g, a.dv - v0 - 8 * g);      // (ahead there is no register for it)
                const f32x8 v = in_f32(next.v);
#pragma unroll
                for (int e = 0; e < 8; ++e) zv += z[e] * v[e];
            }
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const int at = i * THREADS + threadIdx.x, r = at / (COLS / 4), k = 4 * (at % (COLS / 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) dot += next.s[i][e] * next.r[i][e];
                Ss.put4(r, k, next.s[i]);
                Rs.put4(r, k, next.r[i]);
            }
            Us.put4(urow, ucol, next.u);
            ask(c0, min(v0 + ROWS, wide - ROWS));      // (behind the last the same again, for nothing)
            __syncthreads();
            const Of<T, 2> of_z = of<T, 2>(z), of_u = Us.rows(16 * w + r16, 8 * g);
            if (c0 == 0) {
#pragma unroll
                for (int m = 0; m < NP; ++m) {
                    const Of<T, 2> u = Us.rows(16 * (2 * m + half) + r16, 8 * g);
                    X[m] = mma<2>(of_o, u, X[m]);
                    Y[m] = mma22<T>(of_z, u, Y[m]);
                }
            }
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const Of<T, 2> sf = Ss.cols(8 * g, nh + 16 * n, r16), rf = Rs.cols(8 * g, nh + 16 * n, r16);
                oS[n] = mma<2>(of_o, sf, oS[n]);
                zS[n] = mma22<T>(of_z, sf, zS[n]);
                uR[n] = mma22<T>(of_u, rf, uR[n]);
            }
        }

        again();
        const int i0 = 16 * w + 4 * g;      // the lane's first row of the results
        // ---- pairs of tokens; K K^T again, for Y A and its share of dbeta
        if (c0 == 0) {
            bf16x4 pt[NP][3];
#pragma unroll
            for (int m = 0; m < NP; ++m)
#pragma unroll
                for (int q = 0; q < 3; ++q)      // (one in the triangle, where this is not; it is not used there)
                    pt[m][q] = ld4(Pt + ((high_fragment(min(2 * m + half, w), w >> 1) * 3 + q) * 64 + r16 + 16 * (2 * (w & 1) + (g >> 1))) * 8 + 4 * (g & 1));
            zv = sum_of_groups(zv);      // of token 16 w + r16
            f32x4 kk[NP];
#pragma unroll
            for (int m = 0; m < NP; ++m) kk[m] = zero4();
#pragma unroll
            for (int s = 0; s < COLS; s += 32) {
                const int k = s + 8 * g;
                const In<T> ka = frag_rows(Ks, KP, 16 * w + r16, k);
#pragma unroll
                for (int m = 0; m < NP; ++m) kk[m] = mma(ka, frag_rows(Ks, KP, 16 * (2 * m + half) + r16, k), kk[m]);
            }
            for (int k = COLS + 8 * g; k < DK; k += 32) {
                const In<T> ka = fetch<T, FULL>(K + min(16 * w + r16, x.len - 1) * a.kt + k, a.dk - k);
#pragma unroll
                for (int m = 0; m < NP; ++m) kk[m] = mma(ka, fetch<T, FULL>(K + min(16 * (2 * m + half) + r16, x.len - 1) * a.kt + k, a.dk - k), kk[m]);
            }
#pragma unroll
            for (int m = 0; m < NP; ++m) {
                const f32x4 beta = ld_rows(2);
                const int n = 2 * m + half, j = 16 * n + r16;
                f32x4 w1 = zero4(), w2 = zero4();
                if (n <= w) {
                    const float cj = coarse[j], fj = fine[j];
                    f32x4 p = zero4();
#pragma unroll
                    for (int q = 2; q >= 0; --q) p += __builtin_convertvector(pt[m][q], f32x4);
                    f32x4 below;      // of column j's M: from row i on
                    float sum = 0.f;
#pragma unroll
                    for (int e = 3; e >= 0; --e) {
                        const int i = i0 + e;
                        const float D = power(coarse[i] - cj, fine[i] - fj);
                        const bool in = i < x.len;
                        w1[e] = in && j <= i ? D * X[m][e] : 0.f;
                        const float y = in && j < i ? -Y[m][e] * D : 0.f;
                        w2[e] = beta[e] * y;
                        if (j == i) szu[i] = Y[m][e];
                        yk[e] += y * kk[m][e];
                        below[e] = sum += (in && j < i ? X[m][e] * p[e] : 0.f) + w2[e] * kk[m][e];
                    }
                    const float near = __shfl_xor(sum, 16), far = __shfl_xor(sum + near, 32);
                    below += (g & 1 ? 0.f : near) + (g & 2 ? 0.f : far);      // (groups behind)
#pragma unroll
                    for (int e = 0; e < 4; ++e) row[e] += j < i0 + e ? below[e] : 0.f;
                    if (g == 0) scol[w][j] = sum + near + far;
                }
                W1.put4(j, i0, w1);
                W2.put4(j, i0, w2);
            }
            __syncthreads();
            again();
        }

        const f32x4 gamma = ld_rows(0), delta = ld_rows(1), scale = gamma * ld_rows(2);
        // what a row of these products and a row of Q or K have in common; dQ and dK so far
        f32x4 dq[NC], dk[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float k = to_f32(Ks[(i0 + e) * KP + nh + 16 * n + r16]), q = to_f32(Qs[(i0 + e) * KP + nh + 16 * n + r16]);
                oq[e] += oS[n][e] * q;
                uk[e] += uR[n][e] * k;
                zk[e] += zS[n][e] * k;
            }
            dq[n] = gamma * oS[n];
            dk[n] = delta * uR[n] - scale * zS[n];
            __builtin_amdgcn_sched_barrier(0);      // (values of one tile at a time in registers)
        }
        // dQ += W1 K, dK += W1^T Q + W2 K + W2^T K, tokens in steps of 32 (what the triangles leave out is zeros)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            again();
            const int k0 = 32 * t + 8 * g;
            const bool low = t <= w / 2, high = t >= w / 2;
            Of<T, 2> w1, wl, w1t, wu;
            if (low) w1 = W1.cols(k0, 16 * w, r16), wl = W2.cols(k0, 16 * w, r16);
            if (high) w1t = W1.rows(16 * w + r16, k0), wu = W2.rows(16 * w + r16, k0);
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const In<T> k = frag_cols(Ks, KP, k0, nh + 16 * n, r16);
                if (low) dq[n] = mma<2>(w1, k, dq[n]), dk[n] = mma<2>(wl, k, dk[n]);
                if (high) dk[n] = mma<2>(wu, k, dk[n]), dk[n] = mma<2>(w1t, frag_cols(Qs, KP, k0, nh + 16 * n, r16), dk[n]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        again();
        if (share > 1) {      // (these columns of S and R have been read, and no others are written)
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int to = (i0 + e) * DK + c0 + nh + 16 * n + r16;
                    S[to] = dq[n][e];
                    R[to] = dk[n][e];
                }
        } else {
            const long long at = (out_row(a, x.seq, x.tok + i0) * a.Hk + hk) * a.dk + c0 + nh + r16, step = (long long)a.Hk * a.dk;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (i0 + e >= x.len) continue;
                T *q = static_cast<T *>(a.dQ) + at + e * step, *k = static_cast<T *>(a.dK) + at + e * step;
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    if (c0 + nh + 16 * n + r16 < a.dk) q[16 * n] = (T)dq[n][e], k[16 * n] = (T)dk[n][e];
            }
        }
    }

    // ---- beta and the gates
    const int i0 = 16 * w + 4 * g;
    const f32x4 gamma = ld_rows(0), delta = ld_rows(1), beta = ld_rows(2);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        oq[e] = gamma[e] * sum_of_16(oq[e]), uk[e] = delta[e] * sum_of_16(uk[e]), zk[e] = gamma[e] * sum_of_16(zk[e]);
        row[e] = sum_of_16(row[e]), yk[e] = sum_of_16(yk[e]);
        const float zvi = half == 0 ? __shfl(zv, 4 * g + e) : 0.f;
        if (r16 == 0) {
            srow[half][i0 + e] = row[e];
            sstate[half][i0 + e] = oq[e] - beta[e] * zk[e];
            slater[half][i0 + e] = uk[e];
            sbeta[half][i0 + e] = zvi - zk[e] + yk[e];
        }
    }
    dot = sum_of_groups(sum_of_16(dot));
    if (lane == 0) sdot[wave_id()] = vec.gamma[C - 1] * dot;
    __syncthreads();
    if (wave_id() == 0) {      // sums up to the chunk's end, and of the tokens before: u.R k, and M's of each later 16 rows
        float after = lane < x.len ? sstate[0][lane] + sstate[1][lane] : 0.f, before[4] = {slater[0][lane] + slater[1][lane]};
#pragma unroll
        for (int b = 1; b < 4; ++b) before[b] = lane < 16 * b ? scol[b][lane] : 0.f;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const float other = __shfl_down(after, s);
            if (lane + s < 64) after += other;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const float other = __shfl_up(before[b], s);
                if (lane >= s) before[b] += other;
            }
        }
        float e = after + srow[0][lane] + srow[1][lane];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const float sum = __shfl_up(before[b], 1);
            if (lane > 0 && (b == 0 || lane < 16 * b)) e += sum;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) e += sdot[i];
        if (lane < x.len) {
            const long long to = out_row(a, x.seq, x.tok + lane) * a.Hv + h;
            static_cast<T *>(a.dG)[to] = (T)e;
            // u = beta (v - what the state has for k): that difference has been taken, in 24 bits; the other form takes it of sums whose operands have 16.
            // (Below 2^-60 numbers may end before u does.)
            const float beta = rows[2][lane];
            static_cast<T *>(a.dbeta)[to] = (T)(fabsf(beta) > 0x1p-60f ? szu[lane] / beta : sbeta[0][lane] + sbeta[1][lane]);
        }
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

template <typename T, int COLS> void grad(const GDelta &a, dim3 grid, hipStream_t stream)
{
    const uintptr_t values = reinterpret_cast<uintptr_t>(a.V) | reinterpret_cast<uintptr_t>(a.dO) | (uintptr_t)((a.vb | a.vt | a.vh | a.ob | a.ot | a.oh) * sizeof(T));
    gdelta_full(a, sizeof(T)) && a.dv % 32 == 0 && values % 16 == 0 ? grad_kernel<T, COLS, true><<<grid, 512, 0, stream>>>(a)
                                                                   : grad_kernel<T, COLS, false><<<grid, 512, 0, stream>>>(a);
}
template <typename T> hipError_t grad(const GDelta &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((long long)a.chunks * a.Hv));
    a.dk <= 64 ? grad<T, 64>(a, grid, stream) : grad<T, 128>(a, grid, stream);
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
