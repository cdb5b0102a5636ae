// Gated delta rule: the chains over the chunks of a sequence (pf_gdelta.h), forward and backward.  A workgroup of four wavefronts
// has 16 NT rows of a state, [d_v][d_k], for one sequence and value head; its rows are in registers as accumulator tiles of the
// transposed state, tiles of 16 of d_k shared out among the wavefronts, and of everything that runs along the tokens of a chunk a
// wavefront has the 16 tokens 16 w ..
#include "pf_gdelta.h"

namespace pf {
namespace gd {
namespace {

// four values of a state's row from k on
template <bool FULL> __device__ __forceinline__ f32x4 state4(const float *row, int k, int dk)
{
    if constexpr (FULL) {
        return *reinterpret_cast<const f32x4 *>(row + k);
    } else {
        f32x4 v = zero4();
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k + e < dk) v[e] = row[k + e];
        return v;
    }
}
template <bool FULL> __device__ __forceinline__ void state4(float *row, int k, int dk, f32x4 v)
{
    if constexpr (FULL) {
        *reinterpret_cast<f32x4 *>(row + k) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k + e < dk) row[k + e] = v[e];
    }
}

// K or Q of a chunk on its way into LDS
template <typename T, int DK, bool FULL> struct Staged {
    static constexpr int UNITS = C * DK / 8 / 256;
    In<T> r[UNITS];
    __device__ __forceinline__ void load(const T *p, long long step, int len, int dk)
    {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = i * 256 + threadIdx.x, row = u / (DK / 8), k = 8 * (u % (DK / 8));
            r[i] = fetch<T, FULL>(p + min(row, len - 1) * step + k, dk - k);
        }
    }
    __device__ __forceinline__ void store(T *tile) const
    {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = i * 256 + threadIdx.x;
            __builtin_memcpy(__builtin_assume_aligned(tile + u / (DK / 8) * pitch<T>(DK) + 8 * (u % (DK / 8)), 16), &r[i], sizeof(r[i]));
        }
    }
};

// Forward.  OUT: O is wanted; else the states before every chunk and U are kept for the backward.
template <typename T, int DK, int NT, bool FULL, bool OUT>
__global__ __launch_bounds__(256) void scan_kernel(GDelta a)
{
    constexpr int KP = pitch<T>(DK), KS = DK / 32, DT = DK / 64, N = 16 * NT, YP = C + 4;
    typedef Tile<T, 3, N, DK> StateTile;
    typedef Tile<T, 3, N, C> LaterTile;
    typedef Tile<T, 2, N, C> UTile;
    __shared__ __attribute__((aligned(16))) T Ks[2][C * KP];
    __shared__ __attribute__((aligned(16))) char smem[StateTile::kBytes + LaterTile::kBytes + UTile::kBytes + N * YP * 4];
    const StateTile Sp = {reinterpret_cast<T *>(smem)};
    const LaterTile Ud = {reinterpret_cast<T *>(smem + StateTile::kBytes)};
    const UTile Uo = {reinterpret_cast<T *>(smem + StateTile::kBytes + LaterTile::kBytes)};
    float *Yt = reinterpret_cast<float *>(smem + StateTile::kBytes + LaterTile::kBytes + UTile::kBytes);

    // tiles of one head side by side, on one XCD: they read the same K, Q, T and P
    const int tiles = OUT ? (a.dv + N - 1) / N : (a.dv + 31) / 32 * (32 / N);
    const int id = (int)xcd_consecutive(blockIdx.x, gridDim.x), tile = id % tiles, sh = id / tiles;
    const int seq = sh / a.Hv, h = sh - seq * a.Hv, hk = h / (a.Hv / a.Hk), dv0 = tile * N;
    const Sequence q = sequence_at(a, seq);
    const int chunks = (q.len + C - 1) / C;
    const int w = wave_id(), lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;

    int col[NT];      // this lane's rows of the state; those behind d_v are zeros
    bool there[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) col[nt] = min(dv0 + 16 * nt + r16, a.dv - 1), there[nt] = dv0 + 16 * nt + r16 < a.dv;

    f32x4 s[DT][NT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            s[dt][nt] = zero4();
            if (a.S0 && there[nt]) s[dt][nt] = state4<FULL>(a.S0 + ((long long)sh * a.dv + col[nt]) * a.dk, 16 * (w * DT + dt) + 4 * g, a.dk);
        }

    const T *K = static_cast<const T *>(a.K) + seq * a.kb + q.tok * a.kt + hk * a.kh;
    const T *Q = static_cast<const T *>(a.Q) + seq * a.qb + q.tok * a.qt + hk * a.qh;
    const T *V = static_cast<const T *>(a.V) + seq * a.vb + q.tok * a.vt + h * a.vh;
    T *O = static_cast<T *>(a.O);

    Staged<T, DK, FULL> kr;
    In<T> qf[KS];
    T vv[NT][4];
    f32x4 tf[4], gamma, delta, beta;
    f32x8 pf[2];
    float decay = 0.f;
    auto len_of = [&](int c) { return min(C, q.len - C * c); };
    auto load_k = [&](int c) { kr.load(K + (long long)C * c * a.kt, a.kt, len_of(c), a.dk); };
    auto load_q = [&](int c) {
        if constexpr (OUT) {
            const T *p = Q + (C * c + min(16 * w + r16, len_of(c) - 1)) * a.qt;
#pragma unroll
            for (int t = 0; t < KS; ++t) qf[t] = fetch<T, FULL>(p + 32 * t + 8 * g, a.dk - 32 * t - 8 * g);
        }
    };
    auto load_v = [&](int c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const T *p = V + (C * c + min(16 * w + 4 * g + e, len_of(c) - 1)) * a.vt;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) vv[nt][e] = p[col[nt]];
        }
    };
    auto load_t = [&](int c) {
        const float *p = a.T + ((long long)(q.first + c) * a.Hv + h) * kMatrix + (16 * w + r16) * C + 4 * g;
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (b <= w) tf[b] = *reinterpret_cast<const f32x4 *>(p + 16 * b);
    };
    auto load_p = [&](int c) {
        if constexpr (OUT) {
            const float *p = a.P + ((long long)(q.first + c) * a.Hv + h) * kMatrix + (16 * w + r16) * C + 8 * g;
#pragma unroll
            for (int b = 0; b < 2; ++b)
                if (b <= w / 2) pf[b] = *reinterpret_cast<const f32x8 *>(p + 32 * b);
        }
    };
    auto load_vec = [&](int c) {
        const Vec v = vec_at(a.vec, (long long)(q.first + c) * a.Hv + h);
        const int i = 16 * w + 4 * g;
        gamma = *reinterpret_cast<const f32x4 *>(v.gamma + i);
        delta = *reinterpret_cast<const f32x4 *>(v.delta + i);
        beta = *reinterpret_cast<const f32x4 *>(v.beta + i);
        decay = v.gamma[C - 1];
    };
    if (chunks > 0) load_k(0), load_q(0), load_v(0), load_t(0), load_p(0), load_vec(0);

    for (int c = 0; c < chunks; ++c) {
        // (each array's next values are asked for as soon as its present ones are used up)
        const int next = min(c + 1, chunks - 1);
        T *Kc = Ks[c & 1];      // (the other one may still be read)
        kr.store(Kc);
        load_k(next);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) Sp.put4(16 * nt + r16, 16 * (w * DT + dt) + 4 * g, s[dt][nt]);
        if constexpr (!OUT) {
            float *S = a.S + ((long long)(q.first + c) * a.Hv + h) * gdelta_state(a) + dv0 * DK;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f32x4 *>(S + (16 * nt + r16) * DK + 16 * (w * DT + dt) + 4 * g) = s[dt][nt];
        }
        __syncthreads();

        f32x4 m[NT], o[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) m[nt] = o[nt] = zero4();
#pragma unroll
        for (int t = 0; t < KS; ++t) {
            const In<T> kf = frag_rows(Kc, KP, 16 * w + r16, 32 * t + 8 * g);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const Of<T, 3> sp = Sp.rows(16 * nt + r16, 32 * t + 8 * g);
                m[nt] = mma<3>(kf, sp, m[nt]);
                if constexpr (OUT) o[nt] = mma<2>(qf[t], sp, o[nt]);
            }
        }
        load_q(next);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            f32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = beta[e] * ((there[nt] ? to_f32(vv[nt][e]) : 0.f) - gamma[e] * m[nt][e]);
            *reinterpret_cast<f32x4 *>(Yt + (16 * nt + r16) * YP + 16 * w + 4 * g) = y;
            if constexpr (OUT) o[nt] *= gamma;
        }
        load_v(next);
        __syncthreads();

        f32x4 u[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            u[nt] = zero4();
#pragma unroll
            for (int b = 0; b < 4; ++b)
                if (b <= w) u[nt] = mma4(tf[b], *reinterpret_cast<const f32x4 *>(Yt + (16 * nt + r16) * YP + 16 * b + 4 * g), u[nt]);
        }
        load_t(next);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if constexpr (OUT) {
                Uo.put4(16 * nt + r16, 16 * w + 4 * g, u[nt]);
            } else {
                const int wide = (a.dv + 31) / 32 * 32;
                float *U = a.U + (((long long)(q.first + c) * a.Hv + h) * C + 16 * w + 4 * g) * wide + dv0 + 16 * nt + r16;
#pragma unroll
                for (int e = 0; e < 4; ++e) U[e * wide] = u[nt][e];
            }
            Ud.put4(16 * nt + r16, 16 * w + 4 * g, u[nt] * delta);
        }
        const float all = decay;
        load_vec(next);
        __syncthreads();

#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[dt][nt] *= all;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            Of<T, 3> ud[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) ud[nt] = Ud.rows(16 * nt + r16, 32 * t + 8 * g);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const In<T> kt = frag_cols(Kc, KP, 32 * t + 8 * g, 16 * (w * DT + dt), r16);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) s[dt][nt] = mma<3>(kt, ud[nt], s[dt][nt]);
            }
        }
        if constexpr (OUT) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (t <= w / 2) {
                    const Of<T, 2> p = of<T, 2>(pf[t]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) o[nt] = mma22<T>(p, Uo.rows(16 * nt + r16, 32 * t + 8 * g), o[nt]);
                }
            load_p(next);
            const int len = len_of(c);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * w + 4 * g + e;
                    if (there[nt] && i < len) O[(out_row(a, seq, q.tok + C * c + i) * a.Hv + h) * a.dv + col[nt]] = (T)o[nt][e];
                }
        }
    }
    if (!OUT || !a.SL) return;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            if (there[nt]) state4<FULL>(a.SL + ((long long)sh * a.dv + col[nt]) * a.dk, 16 * (w * DT + dt) + 4 * g, a.dk, s[dt][nt]);
}

// Backward, from the last chunk to the first, with R the gradient of the state behind a chunk:
//   dU = P^T dO + delta K R^T ,  Z = T^T dU ,  dV = beta Z ,  R' = gamma_64 R + (gamma dO)^T Q - (gamma beta Z)^T K .
// R and Z are kept for the gradients of Q, K and the gates.
template <typename T, int DK, int NT, bool FULL>
__global__ __launch_bounds__(256) void scan_bwd_kernel(GDelta a)
{
    constexpr int KP = pitch<T>(DK), KS = DK / 32, DT = DK / 64, N = 16 * NT, YP = C + 4;
    typedef Tile<T, 3, N, DK> StateTile;
    typedef Tile<T, 3, N, C> TokenTile;
    // (inputs are held once: the barrier behind a chunk is what that costs)
    __shared__ __attribute__((aligned(16))) T Ks[C * KP], Qs[C * KP];
    __shared__ __attribute__((aligned(16))) char smem[StateTile::kBytes + 2 * TokenTile::kBytes > N * YP * 4 ? StateTile::kBytes + 2 * TokenTile::kBytes : N * YP * 4];
    __shared__ __attribute__((aligned(16))) T dOt[N * pitch<T>(C)];
    const StateTile Rp = {reinterpret_cast<T *>(smem)};
    const TokenTile Dg = {reinterpret_cast<T *>(smem + StateTile::kBytes)};
    const TokenTile Zg = {reinterpret_cast<T *>(smem + StateTile::kBytes + TokenTile::kBytes)};
    float *dUt = reinterpret_cast<float *>(smem);      // in the place of R's parts, once these are used up

    const int wide = (a.dv + 31) / 32 * 32, tiles = wide / N;
    const int id = (int)xcd_consecutive(blockIdx.x, gridDim.x), tile = id % tiles, sh = id / tiles;
    const int seq = sh / a.Hv, h = sh - seq * a.Hv, hk = h / (a.Hv / a.Hk), dv0 = tile * N;
    const Sequence q = sequence_at(a, seq);
    const int chunks = (q.len + C - 1) / C;
    const int w = wave_id(), lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;

    int col[NT];
    bool there[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) col[nt] = min(dv0 + 16 * nt + r16, a.dv - 1), there[nt] = dv0 + 16 * nt + r16 < a.dv;
    f32x4 s[DT][NT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            s[dt][nt] = zero4();
            if (a.dSL && there[nt]) s[dt][nt] = state4<FULL>(a.dSL + ((long long)sh * a.dv + col[nt]) * a.dk, 16 * (w * DT + dt) + 4 * g, a.dk);
        }

    const T *K = static_cast<const T *>(a.K) + seq * a.kb + q.tok * a.kt + hk * a.kh;
    const T *Q = static_cast<const T *>(a.Q) + seq * a.qb + q.tok * a.qt + hk * a.qh;
    const T *dO = static_cast<const T *>(a.dO) + seq * a.ob + q.tok * a.ot + h * a.oh;
    T *dV = static_cast<T *>(a.dV);

    Staged<T, DK, FULL> kr, qr;
    T od[NT][4];
    f32x4 tf[4], gamma, delta, beta;
    f32x8 pf[2];
    float decay = 0.f;
    auto len_of = [&](int c) { return min(C, q.len - C * c); };
    auto load_kq = [&](int c) {
        kr.load(K + (long long)C * c * a.kt, a.kt, len_of(c), a.dk);
        qr.load(Q + (long long)C * c * a.qt, a.qt, len_of(c), a.dk);
    };
    auto load_do = [&](int c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const T *p = dO + (C * c + min(16 * w + 4 * g + e, len_of(c) - 1)) * a.ot;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) od[nt][e] = p[col[nt]];
        }
    };
    // (columns of T and P: rows of their transposes)
    auto load_t = [&](int c) {
        const float *p = a.T + ((long long)(q.first + c) * a.Hv + h) * kMatrix + 4 * g * C + 16 * w + r16;
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (b >= w)
#pragma unroll
                for (int e = 0; e < 4; ++e) tf[b][e] = p[(16 * b + e) * C];
    };
    auto load_p = [&](int c) {
        const float *p = a.P + ((long long)(q.first + c) * a.Hv + h) * kMatrix + 8 * g * C + 16 * w + r16;
#pragma unroll
        for (int b = 0; b < 2; ++b)
            if (b >= w / 2)
#pragma unroll
                for (int e = 0; e < 8; ++e) pf[b][e] = p[(32 * b + e) * C];
    };
    auto load_vec = [&](int c) {
        const Vec v = vec_at(a.vec, (long long)(q.first + c) * a.Hv + h);
        const int i = 16 * w + 4 * g;
        gamma = *reinterpret_cast<const f32x4 *>(v.gamma + i);
        delta = *reinterpret_cast<const f32x4 *>(v.delta + i);
        beta = *reinterpret_cast<const f32x4 *>(v.beta + i);
        decay = v.gamma[C - 1];
    };
    if (chunks > 0) load_kq(chunks - 1), load_do(chunks - 1), load_t(chunks - 1), load_p(chunks - 1), load_vec(chunks - 1);

    for (int c = chunks - 1; c >= 0; --c) {
        const int next = max(c - 1, 0), len = len_of(c);
        const long long x = (long long)(q.first + c) * a.Hv + h;
        kr.store(Ks), qr.store(Qs);
        load_kq(next);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int k = 16 * (w * DT + dt) + 4 * g;
                Rp.put4(16 * nt + r16, k, s[dt][nt]);
                *reinterpret_cast<f32x4 *>(a.R + x * gdelta_state(a) + (dv0 + 16 * nt + r16) * DK + k) = s[dt][nt];
            }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            f32x4 d;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = there[nt] && 16 * w + 4 * g + e < len;
                if (!in) od[nt][e] = (T)0.f;
                d[e] = gamma[e] * to_f32(od[nt][e]);
            }
            __builtin_memcpy(dOt + (16 * nt + r16) * pitch<T>(C) + 16 * w + 4 * g, od[nt], sizeof(od[nt]));
            Dg.put4(16 * nt + r16, 16 * w + 4 * g, d);
        }
        load_do(next);
        __syncthreads();

        f32x4 du[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) du[nt] = zero4();
#pragma unroll
        for (int t = 0; t < KS; ++t) {
            const In<T> kf = frag_rows(Ks, KP, 16 * w + r16, 32 * t + 8 * g);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) du[nt] = mma<3>(kf, Rp.rows(16 * nt + r16, 32 * t + 8 * g), du[nt]);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) du[nt] *= delta;
#pragma unroll
        for (int t = 0; t < 2; ++t)
            if (t >= w / 2) {
                const Of<T, 3> p = of<T, 3>(pf[t]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) du[nt] = mma<3>(p, frag_rows(dOt, pitch<T>(C), 16 * nt + r16, 32 * t + 8 * g), du[nt]);
            }
        load_p(next);
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f32x4 *>(dUt + (16 * nt + r16) * YP + 16 * w + 4 * g) = du[nt];
        __syncthreads();

        f32x4 z[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            z[nt] = zero4();
#pragma unroll
            for (int b = 0; b < 4; ++b)
                if (b >= w) z[nt] = mma4(tf[b], *reinterpret_cast<const f32x4 *>(dUt + (16 * nt + r16) * YP + 16 * b + 4 * g), z[nt]);
        }
        load_t(next);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float *Z = a.Z + (x * C + 16 * w + 4 * g) * wide + dv0 + 16 * nt + r16;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 16 * w + 4 * g + e;
                Z[e * wide] = z[nt][e];
                const float d = beta[e] * z[nt][e];
                if (there[nt] && i < len) dV[(out_row(a, seq, q.tok + C * c + i) * a.Hv + h) * a.dv + col[nt]] = (T)d;
                z[nt][e] = -gamma[e] * d;
            }
            Zg.put4(16 * nt + r16, 16 * w + 4 * g, z[nt]);
        }
        const float all = decay;
        load_vec(next);
        __syncthreads();

#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[dt][nt] *= all;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            Of<T, 3> dg[NT], zg[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) dg[nt] = Dg.rows(16 * nt + r16, 32 * t + 8 * g), zg[nt] = Zg.rows(16 * nt + r16, 32 * t + 8 * g);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const In<T> qt = frag_cols(Qs, KP, 32 * t + 8 * g, 16 * (w * DT + dt), r16);
                const In<T> kt = frag_cols(Ks, KP, 32 * t + 8 * g, 16 * (w * DT + dt), r16);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    s[dt][nt] = mma<3>(qt, dg[nt], s[dt][nt]);
                    s[dt][nt] = mma<3>(kt, zg[nt], s[dt][nt]);
                }
            }
        }
        __syncthreads();
    }
    if (!a.dS0) return;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            if (there[nt]) state4<FULL>(a.dS0 + ((long long)sh * a.dv + col[nt]) * a.dk, 16 * (w * DT + dt) + 4 * g, a.dk, s[dt][nt]);
}

enum { kForward, kKeep, kBackward };

template <typename T, int DK, int NT> hipError_t scan(const GDelta &a, bool full, int what, hipStream_t stream)
{
    const int tiles = what == kForward ? (a.dv + 16 * NT - 1) / (16 * NT) : (a.dv + 31) / 32 * (2 / NT);
    const double groups = (double)a.N * a.Hv * tiles;
    if (!launch_holds(groups, 256)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)groups);
    if (what == kForward)
        full ? scan_kernel<T, DK, NT, true, true><<<grid, 256, 0, stream>>>(a) : scan_kernel<T, DK, NT, false, true><<<grid, 256, 0, stream>>>(a);
    else if (what == kKeep)
        full ? scan_kernel<T, DK, NT, true, false><<<grid, 256, 0, stream>>>(a) : scan_kernel<T, DK, NT, false, false><<<grid, 256, 0, stream>>>(a);
    else
        full ? scan_bwd_kernel<T, DK, NT, true><<<grid, 256, 0, stream>>>(a) : scan_bwd_kernel<T, DK, NT, false><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t scan(const GDelta &a, int what, hipStream_t stream)
{
    const bool full = gdelta_full(a, sizeof(T));
    return a.dk <= 64 ? scan<T, 64, 1>(a, full, what, stream) : a.dk <= 128 ? scan<T, 128, 1>(a, full, what, stream) : scan<T, 256, 1>(a, full, what, stream);
}

}  // namespace
}  // namespace gd

hipError_t launch_gdelta_scan(const GDelta &a, bool is_bf16, bool backward, hipStream_t stream)
{
    const int what = backward ? gd::kKeep : gd::kForward;
    return is_bf16 ? gd::scan<bf16>(a, what, stream) : gd::scan<float>(a, what, stream);
}
hipError_t launch_gdelta_scan_bwd(const GDelta &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? gd::scan<bf16>(a, gd::kBackward, stream) : gd::scan<float>(a, gd::kBackward, stream);
}

}  // namespace pf
