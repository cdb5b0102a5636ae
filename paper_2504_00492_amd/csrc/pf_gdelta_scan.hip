// Gated delta rule: the chains over the chunks of a sequence (pf_gdelta.h), forward and backward.  A workgroup has 16 rows of a state,
// [d_v][d_k], for one sequence and value head.  A chunk's steps come one from the other, and what bounds these kernels is how long they take:
// of 65536 tokens of 32 heads of 128 in bf16 (a workgroup to each compute unit) a chunk takes 2.0 us, 2.05 ms in all; with its inputs
// the same lines every time, so out of the nearest cache, 1.5 us, of which the matrix instructions are about a third and three trips through LDS
// with a barrier each most of the others.  (16 rows: of 32 half as many workgroups, each with longer steps.)
// So eight wavefronts share the work by what waits for what (with four alone the whole call took 3.06 ms, with eight 2.42): four have
// the chain alone, with the state in registers as accumulator tiles of its transpose (tiles of 16 of d_k shared out among them;
// of what runs along the tokens a wavefront has the 16 tokens 16 w ..), and four beside them do all that does not lie in it: they bring
// K into LDS a chunk ahead, and compute the outputs, or in the backward what R does not enter.
#include "pf_gdelta.h"

namespace pf {
namespace gd {
namespace {

constexpr int N = 16;      // rows of a state to a workgroup

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

// K or Q of a chunk.  LDS: by way of it (256 threads bring it there); else, where that has no room, out of memory each time.
template <typename T, int DK, bool FULL, bool LDS> struct Tokens {
    static constexpr int kLd = pitch<T>(DK), kBytes = LDS ? C * kLd * (int)sizeof(T) : 0, UNITS = LDS ? C * DK / 8 / 256 : 1;
    In<T> r[UNITS];
    __device__ __forceinline__ void load(const T *p, long long step, int len, int dk, int thread)
    {
        if constexpr (LDS) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int u = i * 256 + thread, row = u / (DK / 8), k = 8 * (u % (DK / 8));
                r[i] = fetch<T, FULL>(p + min(row, len - 1) * step + k, dk - k);
            }
        }
    }
    __device__ __forceinline__ void store(T *tile, int thread) const
    {
        if constexpr (LDS) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int u = i * 256 + thread;
                __builtin_memcpy(__builtin_assume_aligned(tile + u / (DK / 8) * kLd + 8 * (u % (DK / 8)), 16), &r[i], sizeof(r[i]));
            }
        }
    }
    static __device__ __forceinline__ In<T> row_frag(const T *tile, const T *p, long long step, int len, int dk, int row, int k)
    {
        if constexpr (LDS) return frag_rows(tile, kLd, row, k);
        else return fetch<T, FULL>(p + min(row, len - 1) * step + k, dk - k);
    }
    static __device__ __forceinline__ In<T> cols8(const T *tile, const T *p, long long step, int len, int dk, int k, int n, int half, int r16)
    {
        if constexpr (LDS) {
            return frag_cols8(tile, kLd, k, n, half, r16);
        } else {
            In<T> f;
            const int c = n + 8 * (r16 >> 2) + 4 * half + (r16 & 3);
#pragma unroll
            for (int e = 0; e < 8; ++e) f.v[e] = FULL || c < dk ? p[min(k + e, len - 1) * step + c] : (T)0.f;
            return f;
        }
    }
};

// The parts of a matrix of pairs: what rows 16 w .. have of its triangle (LOW: up to the diagonal, else from it on), `lane` the lane's place
// in a fragment.
template <int NP, bool LOW> struct Pairs {
    Of<bf16, NP> f[2];
    __device__ __forceinline__ void load(const bf16 *p, int w, int lane)
    {
        p += (LOW ? low_fragment(w, 0) : high_fragment(w, w >> 1)) * 3 * 512 + lane * 8;
#pragma unroll
        for (int i = 0; i < NP; ++i) f[LOW ? 0 : 1].p[i] = ld8(p + i * 512 + (LOW ? 0 : w < 2 ? 3 * 512 : 0));
        if (LOW ? w >= 2 : w < 2)
#pragma unroll
            for (int i = 0; i < NP; ++i) f[LOW ? 1 : 0].p[i] = ld8(p + i * 512 + (LOW ? 3 * 512 : 0));
    }
};

struct Place {      // of a workgroup: its sequence, head and first row of the state; its segment, whose tokens and chunks q has
    int seq, h, hk, dv0, chunks, seg;
    Sequence q;
    long long sh, at;      // at: of the segment among all
};
__device__ __forceinline__ Place place_of(const GDelta &a, int tiles)
{
    // tiles of one head side by side, on one XCD: they read the same K, Q, T and P
    Place x;
    const int id = uniform((int)xcd_consecutive(blockIdx.x, gridDim.x)), all = id / tiles, sh = all / a.segments;
    x.sh = sh, x.at = all, x.seg = all - sh * a.segments;
    x.seq = sh / a.Hv, x.h = sh - x.seq * a.Hv, x.hk = x.h / (a.Hv / a.Hk), x.dv0 = (id - all * tiles) * N;
    x.q = sequence_at(a, x.seq);
    x.chunks = (x.q.len + C - 1) / C;
    if (a.segments > 1) {
        const int from = (int)((long long)x.chunks * x.seg / a.segments), to = (int)((long long)x.chunks * (x.seg + 1) / a.segments);
        x.q = {x.q.tok + C * from, min(x.q.len, C * to) - C * from, x.q.first + from};
        x.chunks = to - from;
    }
    return x;
}
__device__ __forceinline__ int wide_of(const GDelta &a) { return (a.dv + 31) / 32 * 32; }

// What a wavefront of the chain has of the state: SLABS times 32 of d_k, from 32 SLABS w on (d_k = 64: two of the four have any), as it
// comes out of the products with the tokens and goes into the next: a lane has the eight neighbours 8 g .. of its row.
template <int DK> struct Share {
    static constexpr int SLABS = DK <= 128 ? 1 : DK / 128, HOLDERS = DK / 32 / SLABS;
};
template <bool FULL, int SLABS> __device__ __forceinline__ void get_state(const float *row, int k, int dk, f32x8 (&s)[SLABS])
{
#pragma unroll
    for (int i = 0; i < SLABS; ++i) {
        const f32x4 a = state4<FULL>(row, k + 32 * i, dk), b = state4<FULL>(row, k + 32 * i + 4, dk);
        s[i] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}
template <bool FULL, int SLABS> __device__ __forceinline__ void put_state(float *row, int k, int dk, const f32x8 (&s)[SLABS])
{
#pragma unroll
    for (int i = 0; i < SLABS; ++i) {
        state4<FULL>(row, k + 32 * i, dk, __builtin_shufflevector(s[i], s[i], 0, 1, 2, 3));
        state4<FULL>(row, k + 32 * i + 4, dk, __builtin_shufflevector(s[i], s[i], 4, 5, 6, 7));
    }
}

// Fragments of a chunk's tokens for a wavefront of the chain: for each of its 32 of d_k the rows of the four tiles of 16 tokens, counted from its
// own (w ^ i), so that registers are named at compile time; and the columns, of the first and the last 32 tokens.
template <typename T, int SLABS> struct Fragments {
    In<T> f[SLABS][4];
    template <typename K> __device__ __forceinline__ void rows(const T *tile, const T *p, long long step, int len, int dk, int w, int lane)
    {
        const int r16 = lane & 15, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < SLABS; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) f[t][i] = K::row_frag(tile, p, step, len, dk, 16 * (w ^ i) + r16, 32 * (w * SLABS + t) + 8 * g);
    }
    template <typename K> __device__ __forceinline__ void cols(const T *tile, const T *p, long long step, int len, int dk, int w, int lane)
    {
        const int r16 = lane & 15, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < SLABS; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) f[t][i] = K::cols8(tile, p, step, len, dk, 32 * (i >> 1) + 8 * g, 32 * (w * SLABS + t), i & 1, r16);
    }
};

// Tokens times the transposed state: each holder multiplies what it has of d_k for all 64 tokens; the others' parts go through LDS (1 KB
// as the lanes hold it).
template <typename T, int DK>
__device__ __forceinline__ f32x4 products(const Fragments<T, Share<DK>::SLABS> &k, const Of<T, 3> (&sp)[Share<DK>::SLABS], f32x4 *parts, int w, int lane)
{
    f32x4 m[4] = {zero4(), zero4(), zero4(), zero4()};
    if (w < Share<DK>::HOLDERS) {
#pragma unroll
        for (int t = 0; t < Share<DK>::SLABS; ++t) mma_each(k.f[t], sp[t], m);
#pragma unroll
        for (int i = 1; i < 4; ++i) parts[((w ^ i) * 3 + i - 1) * 64 + lane] = m[i];
    }
    return m[0];
}
template <int DK> __device__ __forceinline__ f32x4 joined(f32x4 own, const f32x4 *parts, int w, int lane)
{
    const f32x4 *p = parts + w * 3 * 64 + lane;
    if constexpr (Share<DK>::HOLDERS == 4) return (own + p[0]) + (p[64] + p[128]);
    else return w < 2 ? own + p[0] : p[64] + p[128];
}
// s = all s + (h, if any) + tokens^T x, x[2] of the first and the last 32 tokens
template <typename T, int SLABS>
__device__ __forceinline__ void update(f32x8 (&s)[SLABS], float all, const f32x4 *h, const Fragments<T, SLABS> &k, const Of<T, 3> (&x)[2])
{
#pragma unroll
    for (int t = 0; t < SLABS; ++t) {
        f32x4 n[2] = {__builtin_shufflevector(s[t], s[t], 0, 1, 2, 3) * all, __builtin_shufflevector(s[t], s[t], 4, 5, 6, 7) * all}, l[2] = {zero4(), zero4()};
        if (h) l[0] = h[t * 128], l[1] = h[t * 128 + 64];
        const In<T> a[2] = {k.f[t][0], k.f[t][1]}, b[2] = {k.f[t][2], k.f[t][3]};
        mma_each(a, x[0], n);
        mma_each(b, x[1], l);
        s[t] = stack(n[0] + l[0], n[1] + l[1]);
    }
}
// Four neighbouring values of a row of the outputs, of which `left` are there.  WHOLE: rows are whole and lie at multiples of their size.
template <typename T> __device__ __forceinline__ void put_row(T *to, f32x4 v, int left, bool whole)
{
    typedef T t4 __attribute__((ext_vector_type(4)));
    if (whole) {
        *reinterpret_cast<t4 *>(to) = __builtin_convertvector(v, t4);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) to[e] = (T)v[e];
    }
}

enum { kForward, kKeep, kEnds, kBackward };

// Forward.  kForward: O is wanted; kKeep: the states before every chunk and U are kept for the backward; kEnds: the states behind each segment alone,
// from zeros, and in d_k more rows what a segment makes of the unit matrix (with no values).
template <typename T, int DK, bool FULL, int WHAT>
__global__ __launch_bounds__(512) void scan_kernel(GDelta a)
{
    constexpr bool OUT = WHAT == kForward;
    constexpr int KS = DK / 32, NPO = sizeof(T) == 2 ? 2 : 3, SLABS = Share<DK>::SLABS, UP = C + 4;      // NPO: parts on the way into O
    typedef Tile<T, NPO, N, DK> StateTile;
    typedef Tile<T, 3, N, C> LaterTile;
    typedef Tile<bf16, 3, N, C> YTile;
    constexpr int kWork = (OUT ? StateTile::kBytes : 0) + LaterTile::kBytes + YTile::kBytes + N * UP * 4 + (12 + 4) * 1024 + 4 * C * 4;
    typedef Tokens<T, DK, FULL, 2 * C * pitch<T>(DK) * (int)sizeof(T) + kWork <= 160 * 1024> KTile;
    __shared__ __attribute__((aligned(16))) char smem[2 * KTile::kBytes + kWork];
    char *at = smem + 2 * KTile::kBytes;
    auto take = [&](int bytes) { char *p = at; at += bytes; return p; };
    f32x4 *parts = reinterpret_cast<f32x4 *>(take(12 * 1024)), *bv = reinterpret_cast<f32x4 *>(take(4 * 1024));      // bv: beta v
    float *rate = reinterpret_cast<float *>(take(4 * C * 4));      // beta gamma, -, delta of even and odd chunks
    const LaterTile Ud = {reinterpret_cast<T *>(take(LaterTile::kBytes))};
    const YTile Yp = {reinterpret_cast<bf16 *>(take(YTile::kBytes))};
    float *Uf = reinterpret_cast<float *>(take(N * UP * 4));
    const StateTile Sp = {reinterpret_cast<T *>(at)};
    auto k_tile = [&](int c) { return reinterpret_cast<T *>(smem + (c & 1) * KTile::kBytes); };

    const Place x = place_of(a, OUT ? (a.dv + N - 1) / N : (wide_of(a) + (WHAT == kEnds ? DK : 0)) / N);
    const int w = wave_id() & 3, lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4, i0 = 16 * w + 4 * g;
    const int col = min(x.dv0 + r16, a.dv - 1);      // this lane's row of the state; those behind d_v are zeros
    const bool there = x.dv0 + r16 < a.dv;
    const T *K = static_cast<const T *>(a.K) + x.seq * a.kb + x.q.tok * a.kt + x.hk * a.kh;
    const long long first = (long long)x.q.first * a.Hv + x.h;
    auto len_of = [&](int c) { return min(C, x.q.len - C * c); };

    if (wave_id() >= 4) {      // ---- beside the chain
        const int thread = threadIdx.x - 256, wide = wide_of(a);
        const T *Q = static_cast<const T *>(a.Q) + x.seq * a.qb + x.q.tok * a.qt + x.hk * a.qh;
        const T *V = static_cast<const T *>(a.V) + x.seq * a.vb + x.q.tok * a.vt + x.h * a.vh + col;
        // O of token 16 w + r16, rows 4 g .. of the 16
        const int t0 = 16 * w + r16, left = a.dv - x.dv0 - 4 * g;      // (or U's)
        const bool whole = a.dv % 4 == 0;
        T *O = static_cast<T *>(a.O) + ((out_row(a, x.seq, x.q.tok) + t0) * a.Hv + x.h) * a.dv + x.dv0 + 4 * g;
        KTile kr;
        In<T> qf[KS];
        T vv[4];
        Pairs<NPO, true> pf;
        f32x4 gamma, beta, delta;
        float since = 0.f;
        auto load = [&](int c) {      // what the chain takes
            kr.load(K + (long long)C * c * a.kt, a.kt, len_of(c), a.dk, thread);
            const T *p = V + (long long)C * c * a.vt;
            const int len = len_of(c);
#pragma unroll
            for (int e = 0; e < 4; ++e) vv[e] = p[min(i0 + e, len - 1) * a.vt];
            const Vec v = vec_at(a.vec, first + (long long)c * a.Hv);
            gamma = *reinterpret_cast<const f32x4 *>(v.gamma + i0);
            delta = *reinterpret_cast<const f32x4 *>(v.delta + i0);
            beta = *reinterpret_cast<const f32x4 *>(v.beta + i0);
        };
        auto store = [&](int c) {
            kr.store(k_tile(c), thread);
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = there ? beta[e] * to_f32(vv[e]) : 0.f;
            bv[w * 64 + lane] = v;
            if (r16 == 0) {
                *reinterpret_cast<f32x4 *>(rate + i0) = beta * gamma;
                *reinterpret_cast<f32x4 *>(rate + (2 + (c & 1)) * C + i0) = delta;
                if (w == 3 && g == 3) rate[C + (c & 1)] = gamma[3];      // of the chunk's end
            }
        };
        auto load_q = [&](int c) {
            const T *p = Q + (C * c + min(16 * w + r16, len_of(c) - 1)) * a.qt;
#pragma unroll
            for (int t = 0; t < KS; ++t) qf[t] = fetch<T, FULL>(p + 32 * t + 8 * g, a.dk - 32 * t - 8 * g);
            since = vec_at(a.vec, first + (long long)c * a.Hv).gamma[t0];
        };
        auto load_p = [&](int c) { pf.load(a.P + (first + (long long)c * a.Hv) * kMatrix, w, lane); };
        if (x.chunks > 0) {
            load(0);
            if constexpr (OUT) load_q(0), load_p(0);
            store(0);
            load(min(1, x.chunks - 1));
        }
        __syncthreads();
        for (int c = 0; c < x.chunks; ++c) {
            const int next = min(c + 1, x.chunks - 1);
            __syncthreads();      // parts of K S^T, and S for O
            f32x4 o[2] = {zero4(), zero4()};
            if constexpr (OUT) {
#pragma unroll
                for (int t = 0; t < KS; ++t) o[t & 1] = mma<NPO>(Sp.rows(r16, 32 * t + 8 * g), qf[t], o[t & 1]);
                o[0] = (o[0] + o[1]) * since;
                load_q(next);
            }
            __syncthreads();      // Y
            store(c + 1);
            load(min(c + 2, x.chunks - 1));
            __syncthreads();      // U
            if constexpr (OUT) {
                auto u = [&](int t) {
                    f32x8 v;
                    __builtin_memcpy(&v, __builtin_assume_aligned(Uf + r16 * UP + 32 * t + 8 * g, 16), sizeof(v));
                    return of<bf16, NPO>(v);
                };
                o[1] = mma_parts<NPO>(u(0), pf.f[0], zero4());
                if (w >= 2) o[0] = mma_parts<NPO>(u(1), pf.f[1], o[0]);
                load_p(next);
                if (t0 < len_of(c) && left > 0) put_row(O + (long long)C * c * a.Hv * a.dv, o[0] + o[1], left, whole);
            } else if constexpr (WHAT == kKeep) {
                const float *u = Uf + 4 * g * UP + t0;
                *reinterpret_cast<f32x4 *>(a.U + ((first + (long long)c * a.Hv) * C + t0) * wide + x.dv0 + 4 * g) = f32x4{u[0], u[UP], u[2 * UP], u[3 * UP]};
            }
        }
        return;
    }

    // ---- the chain
    const bool holds = w < Share<DK>::HOLDERS;
    const int k0 = 32 * w * SLABS + 8 * g;
    f32x8 s[SLABS];
#pragma unroll
    for (int t = 0; t < SLABS; ++t) s[t] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int wide = wide_of(a);
    if constexpr (WHAT == kEnds) {
#pragma unroll
        for (int t = 0; t < SLABS; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[t][e] = x.dv0 + r16 == wide + k0 + 32 * t + e ? 1.f : 0.f;
    } else if (a.segments > 1) {
        if (holds) get_state<true>(a.starts + (x.at * wide + x.dv0 + r16) * DK, k0, DK, s);
    } else if (a.S0 && there && holds) {
        get_state<FULL>(a.S0 + (x.sh * a.dv + col) * a.dk, k0, a.dk, s);
    }
    Pairs<3, true> tf;
    auto load_t = [&](int c) { tf.load(a.T + (first + (long long)c * a.Hv) * kMatrix, w, lane); };
    if (x.chunks > 0) load_t(0);
    __syncthreads();
    Fragments<T, SLABS> kf, kc;
    auto rows = [&](int c) { kf.template rows<KTile>(k_tile(c), K + (long long)C * c * a.kt, a.kt, len_of(c), a.dk, w, lane); };
    auto cols = [&](int c) { kc.template cols<KTile>(k_tile(c), K + (long long)C * c * a.kt, a.kt, len_of(c), a.dk, w, lane); };
    constexpr bool AHEAD = KTile::kBytes > 0;      // (out of memory they are taken where they are used: there are no registers for more)
    if (AHEAD && x.chunks > 0 && holds) rows(0);

    for (int c = 0; c < x.chunks; ++c) {
        if (!AHEAD && holds) rows(c);
        Of<T, 3> sp[SLABS];
#pragma unroll
        for (int t = 0; t < SLABS; ++t) sp[t] = of<T, 3>(s[t]);
        const f32x4 own = products<T, DK>(kf, sp, parts, w, lane);
        if (holds) {
            if constexpr (OUT) {
#pragma unroll
                for (int t = 0; t < SLABS; ++t) Sp.put8(r16, k0 + 32 * t, sp[t]);
            } else if constexpr (WHAT == kKeep) {
                put_state<true>(a.S + (first + (long long)c * a.Hv) * gdelta_state(a) + (x.dv0 + r16) * DK, k0, DK, s);
            }
        }
        __syncthreads();

        const f32x4 m = joined<DK>(own, parts, w, lane);
        Yp.put4(r16, i0, bv[w * 64 + lane] - *reinterpret_cast<const f32x4 *>(rate + i0) * m);
        __syncthreads();

        f32x4 u = mma33(tf.f[0], Yp.rows(r16, 8 * g), zero4());
        if (w >= 2) u += mma33(tf.f[1], Yp.rows(r16, 32 + 8 * g), zero4());
        load_t(min(c + 1, x.chunks - 1));
        Ud.put4(r16, i0, u * *reinterpret_cast<const f32x4 *>(rate + (2 + (c & 1)) * C + i0));
        *reinterpret_cast<f32x4 *>(Uf + r16 * UP + i0) = u;
        const float all = rate[C + (c & 1)];
        if (AHEAD && holds) cols(c);
        __syncthreads();

        if (holds) {
            const Of<T, 3> ud[2] = {Ud.rows(r16, 8 * g), Ud.rows(r16, 32 + 8 * g)};
            if (!AHEAD) cols(c);
            else if (c + 1 < x.chunks) rows(c + 1);
            update<T, SLABS>(s, all, nullptr, kc, ud);
        }
    }
    if (WHAT == kEnds && holds) put_state<true>(a.ends + (x.at * (wide + DK) + x.dv0 + r16) * DK, k0, DK, s);
    if (OUT && a.SL && there && holds && x.seg == a.segments - 1) put_state<FULL>(a.SL + (x.sh * a.dv + col) * a.dk, k0, a.dk, s);
}

// Backward, from the last chunk to the first, with R the gradient of the state behind a chunk:
//   dU = P^T dO + delta K R^T ,  Z = T^T dU ,  dV = beta Z ,  R' = gamma_64 R + (gamma dO)^T Q - (gamma beta Z)^T K .
// ends: R in front of each segment alone, from zeros (what else is written is written again behind that).
// R and Z are kept for the gradients of Q, K and the gates.  P^T dO and (gamma dO)^T Q are computed beside the chain, a chunk ahead.
template <typename T, int DK, bool FULL, int GROUPS>
__global__ __launch_bounds__(256 * GROUPS) void scan_bwd_kernel(GDelta a, bool ends)
{
    constexpr int OP = pitch<T>(C), XP = C + 4, SLABS = Share<DK>::SLABS, HOLDERS = Share<DK>::HOLDERS;
    typedef Tile<T, 3, N, C> TokenTile;
    typedef Tile<bf16, 3, N, C> DUTile;
    constexpr int kQd = HOLDERS * SLABS * 2 * 1024;
    constexpr int kWork = 2 * TokenTile::kBytes + DUTile::kBytes + N * OP * (int)sizeof(T) + kQd + (12 + 4) * 1024 + N * XP * 4 + 4 * C * 4;
    constexpr int kOne = C * pitch<T>(DK) * (int)sizeof(T);
    typedef Tokens<T, DK, FULL, 2 * kOne + kWork <= 160 * 1024> KTile;
    typedef Tokens<T, DK, FULL, 3 * kOne + kWork <= 160 * 1024> QTile;
    __shared__ __attribute__((aligned(16))) char smem[2 * KTile::kBytes + QTile::kBytes + kWork];
    char *at = smem + 2 * KTile::kBytes + QTile::kBytes;
    auto take = [&](int bytes) { char *p = at; at += bytes; return p; };
    f32x4 *parts = reinterpret_cast<f32x4 *>(take(12 * 1024)), *pd = reinterpret_cast<f32x4 *>(take(4 * 1024));      // pd: P^T dO
    f32x4 *qd = reinterpret_cast<f32x4 *>(take(kQd));                // (gamma dO)^T Q
    float *zf = reinterpret_cast<float *>(take(N * XP * 4));           // Z, turned
    float *rate = reinterpret_cast<float *>(take(4 * C * 4));      // delta, gamma_64, gamma beta of even and odd chunks
    const TokenTile Dg = {reinterpret_cast<T *>(take(TokenTile::kBytes))}, Zg = {reinterpret_cast<T *>(take(TokenTile::kBytes))};
    const DUTile Du = {reinterpret_cast<bf16 *>(take(DUTile::kBytes))};
    T *dOt = reinterpret_cast<T *>(at);      // dO, turned
    auto k_tile = [&](int c) { return reinterpret_cast<T *>(smem + (c & 1) * KTile::kBytes); };
    T *Qs = reinterpret_cast<T *>(smem + 2 * KTile::kBytes);

    const int wide = wide_of(a);
    const Place x = place_of(a, wide / N);
    const int w = wave_id() & 3, lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4, i0 = 16 * w + 4 * g;
    const int col = min(x.dv0 + r16, a.dv - 1);
    const bool there = x.dv0 + r16 < a.dv, holds = w < HOLDERS;
    const T *K = static_cast<const T *>(a.K) + x.seq * a.kb + x.q.tok * a.kt + x.hk * a.kh;
    const long long first = (long long)x.q.first * a.Hv + x.h;
    const int last = x.chunks - 1;
    auto len_of = [&](int c) { return min(C, x.q.len - C * c); };

    if (wave_id() >= 4) {      // ---- beside the chain
        const int thread = threadIdx.x & 255;
        const bool carry = GROUPS == 2 || wave_id() < 8, read = GROUPS == 2 || wave_id() >= 8;
        const T *Q = static_cast<const T *>(a.Q) + x.seq * a.qb + x.q.tok * a.qt + x.hk * a.qh;
        const T *dO = static_cast<const T *>(a.dO) + x.seq * a.ob + x.q.tok * a.ot + x.h * a.oh + col;
        const int t0 = 16 * w + r16, left = a.dv - x.dv0 - 4 * g;      // Z and dV of this token, rows 4 g .. of the 16
        const bool whole = a.dv % 4 == 0;
        T *dV = static_cast<T *>(a.dV) + ((out_row(a, x.seq, x.q.tok) + t0) * a.Hv + x.h) * a.dv + x.dv0 + 4 * g;
        KTile kr;
        QTile qr;
        T od[4];
        f32x4 gamma, delta, beta;
        float rate_of = 0.f, next_rate = 0.f, now = 0.f;      // beta of this lane's token: as loaded, and of the next two chunks to be stored
        f32x4 z = zero4();
        // Z and dV are stored at once, or by a group of their own a chunk later: memory answers in order, so what waits for its loads of P
        // waits for the stores before them, which are a chunk old then (both at d = 128: 491 -> 373 us; of two groups, d = 64: 64 and 82).
        constexpr bool LATER = GROUPS == 3;
        auto put = [&](int c) {
            *reinterpret_cast<f32x4 *>(a.Z + ((first + (long long)c * a.Hv) * C + t0) * wide + x.dv0 + 4 * g) = z;
            if (t0 < len_of(c) && left > 0) put_row(dV + (long long)C * c * a.Hv * a.dv, now * z, left, whole);
        };
        Pairs<3, false> pf;
        f32x4 p = zero4(), h[SLABS][2];
        auto load = [&](int c) {
            const int len = len_of(c);
            kr.load(K + (long long)C * c * a.kt, a.kt, len, a.dk, thread);
            qr.load(Q + (long long)C * c * a.qt, a.qt, len, a.dk, thread);
            const T *o = dO + (long long)C * c * a.ot;
#pragma unroll
            for (int e = 0; e < 4; ++e) od[e] = o[min(i0 + e, len - 1) * a.ot];
            const Vec v = vec_at(a.vec, first + (long long)c * a.Hv);
            gamma = *reinterpret_cast<const f32x4 *>(v.gamma + i0);
            delta = *reinterpret_cast<const f32x4 *>(v.delta + i0);
            beta = *reinterpret_cast<const f32x4 *>(v.beta + i0);
        };
        auto load_p = [&](int c) {
            pf.load(a.P + (first + (long long)c * a.Hv) * kMatrix, w, lane);
            rate_of = vec_at(a.vec, first + (long long)c * a.Hv).beta[t0];
        };
        auto store = [&](int c) {
            kr.store(k_tile(c), thread), qr.store(Qs, thread);
            const int len = len_of(c);
            f32x4 d;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (!there || i0 + e >= len) od[e] = (T)0.f;
                d[e] = gamma[e] * to_f32(od[e]);
            }
            __builtin_memcpy(dOt + r16 * OP + i0, od, sizeof(od));
            Dg.put4(r16, i0, d);
            if (r16 == 0) {
                *reinterpret_cast<f32x4 *>(rate + i0) = delta;
                *reinterpret_cast<f32x4 *>(rate + (2 + (c & 1)) * C + i0) = -gamma * beta;
                if (w == 3 && g == 3) rate[C + (c & 1)] = gamma[3];
            }
        };
        auto multiply = [&](int c) {
            const T *Qg = Q + (long long)C * c * a.qt;
            const int len = len_of(c);
            p = zero4();
            if (w < 2) p = mma_input(pf.f[0], frag_rows(dOt, OP, r16, 8 * g), p);
            p = mma_input(pf.f[1], frag_rows(dOt, OP, r16, 32 + 8 * g), p);
            if (!holds) return;
#pragma unroll
            for (int t = 0; t < SLABS; ++t) {
                h[t][0] = h[t][1] = zero4();
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const Of<T, 3> d = Dg.rows(r16, 32 * b + 8 * g);
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        h[t][half] = mma<3>(QTile::cols8(Qs, Qg, a.qt, len, a.dk, 32 * b + 8 * g, 32 * (w * SLABS + t), half, r16), d, h[t][half]);
                }
            }
        };
        if (last >= 0 && read) load_p(last);
        if (last >= 0 && carry) {
            load(last);
            store(last);
            load(max(last - 1, 0));
        }
        __syncthreads();
        if (last >= 0 && read) {
            multiply(last);
            now = next_rate = rate_of;
            load_p(max(last - 1, 0));
            pd[w * 64 + lane] = p;
        }
        __syncthreads();
        for (int c = last; c >= 0; --c) {
            const int next = max(c - 1, 0);      // (before the first chunk the same again, which nobody takes)
            __syncthreads();      // parts of K R^T
            if (holds && read) {
#pragma unroll
                for (int t = 0; t < SLABS; ++t)
#pragma unroll
                    for (int half = 0; half < 2; ++half) qd[((w * SLABS + t) * 2 + half) * 64 + lane] = h[t][half];
            }
            __syncthreads();      // dU
            if (carry && c > 0) store(next);
            if (LATER && read) {
                if (c < last) put(c + 1);
                now = next_rate, next_rate = rate_of;
            }
            if (carry) load(max(c - 2, 0));
            __syncthreads();      // Z
            if (!read) continue;
            const float *q = zf + 4 * g * XP + t0;
            z = f32x4{q[0], q[XP], q[2 * XP], q[3 * XP]};
            if constexpr (!LATER) {
                put(c);
                now = rate_of;
            }
            multiply(next);
            load_p(max(c - 2, 0));
            pd[w * 64 + lane] = p;
        }
        if (LATER && read && last >= 0) put(0);
        return;
    }

    // ---- the chain
    const int k0 = 32 * w * SLABS + 8 * g;
    f32x8 s[SLABS];
#pragma unroll
    for (int t = 0; t < SLABS; ++t) s[t] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.segments > 1) {
        if (holds && !ends) get_state<true>(a.starts + (x.at * wide + x.dv0 + r16) * DK, k0, DK, s);
    } else if (a.dSL && there && holds) {
        get_state<FULL>(a.dSL + (x.sh * a.dv + col) * a.dk, k0, a.dk, s);
    }
    Pairs<3, false> tf;
    auto load_t = [&](int c) { tf.load(a.Tt + (first + (long long)c * a.Hv) * kMatrix, w, lane); };
    if (last >= 0) load_t(last);
    __syncthreads();
    __syncthreads();
    Fragments<T, SLABS> kf, kc;
    auto rows = [&](int c) { kf.template rows<KTile>(k_tile(c), K + (long long)C * c * a.kt, a.kt, len_of(c), a.dk, w, lane); };
    auto cols = [&](int c) { kc.template cols<KTile>(k_tile(c), K + (long long)C * c * a.kt, a.kt, len_of(c), a.dk, w, lane); };
    constexpr bool AHEAD = KTile::kBytes > 0;      // (as in the forward)
    if (AHEAD && last >= 0 && holds) rows(last);

    for (int c = last; c >= 0; --c) {
        if (!AHEAD && holds) rows(c);
        Of<T, 3> sp[SLABS];
#pragma unroll
        for (int t = 0; t < SLABS; ++t) sp[t] = of<T, 3>(s[t]);
        const f32x4 own = products<T, DK>(kf, sp, parts, w, lane);
        if (holds) put_state<true>(a.R + (first + (long long)c * a.Hv) * gdelta_state(a) + (x.dv0 + r16) * DK, k0, DK, s);
        __syncthreads();

        Du.put4(r16, i0, joined<DK>(own, parts, w, lane) * *reinterpret_cast<const f32x4 *>(rate + i0) + pd[w * 64 + lane]);
        __syncthreads();

        f32x4 z = mma33(tf.f[1], Du.rows(r16, 32 + 8 * g), zero4());
        if (w < 2) z += mma33(tf.f[0], Du.rows(r16, 8 * g), zero4());
        load_t(max(c - 1, 0));
        Zg.put4(r16, i0, z * *reinterpret_cast<const f32x4 *>(rate + (2 + (c & 1)) * C + i0));
        *reinterpret_cast<f32x4 *>(zf + r16 * XP + i0) = z;
        const float all = rate[C + (c & 1)];
        if (AHEAD && holds) cols(c);
        __syncthreads();

        if (holds) {
            const Of<T, 3> zg[2] = {Zg.rows(r16, 8 * g), Zg.rows(r16, 32 + 8 * g)};
            if (!AHEAD) cols(c);
            else if (c > 0) rows(c - 1);
            update<T, SLABS>(s, all, qd + w * SLABS * 128 + lane, kc, zg);
        }
    }
    if (ends) {
        if (holds) put_state<true>(a.fronts + (x.at * wide + x.dv0 + r16) * DK, k0, DK, s);
    } else if (a.dS0 && there && holds && x.seg == 0) {
        put_state<FULL>(a.dS0 + (x.sh * a.dv + col) * a.dk, k0, a.dk, s);
    }
}

// States at the ends of segments, one segment after the other, S <- S M + L with M what the segment makes of the unit matrix and L its state from
// zeros; BACK: gradients, from the last on, R <- R M^T + L.  A workgroup has 16 rows of a state, a wavefront 16 columns of it; a step's M is asked
// for a step ahead.
template <int DK, bool BACK> __global__ __launch_bounds__(4 * DK) void join_kernel(GDelta a)
{
    constexpr int STEPS = DK / 4, P = DK + 4;
    __shared__ __attribute__((aligned(16))) float state[2][16 * P];
    const int wide = wide_of(a), tiles = wide / N, w = wave_id(), lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
    const long long sh = blockIdx.x / tiles;
    const int dv0 = (int)(blockIdx.x - sh * tiles) * N, col = 16 * w + r16;
    const float *first = BACK ? a.dSL : a.S0;
    f32x4 s;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int row = dv0 + 4 * g + e;
        s[e] = first && row < a.dv && col < a.dk ? first[(sh * a.dv + row) * a.dk + col] : 0.f;
    }
    f32x4 m[STEPS / 4];      // of its column, every fourth row from g on (BACK: of M^T the rows from STEPS g on, in whole vectors)
    f32x4 l;
    const uint32_t mine = g * DK + col;      // (beside an address that is the same for all lanes)
    auto ask = [&](int seg) {
        const long long at = sh * a.segments + seg;
        const float *M = a.ends + (at * (wide + DK) + wide) * DK, *L = BACK ? a.fronts + (at * wide + dv0 + 4 * g) * DK + col : a.ends + (at * (wide + DK) + dv0 + 4 * g) * DK + col;
#pragma unroll
        for (int i = 0; i < STEPS / 4; ++i) {
            if constexpr (BACK) m[i] = *reinterpret_cast<const f32x4 *>(M + col * DK + STEPS * g + 4 * i);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) m[i][e] = (M + 4 * (4 * i + e) * DK)[mine];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) l[e] = L[e * DK];
    };
    ask(BACK ? a.segments - 1 : 0);
    for (int i = 0; i < a.segments; ++i) {
        const int seg = BACK ? a.segments - 1 - i : i;
        float *now = state[i & 1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a.starts[((sh * a.segments + seg) * wide + dv0 + 4 * g + e) * DK + col] = s[e];
            now[(4 * g + e) * P + col] = s[e];
        }
        __syncthreads();
        f32x4 n[2] = {l, zero4()};
#pragma unroll
        for (int i = 0; i < STEPS / 4; ++i) {
            f32x4 x;
            if constexpr (BACK) x = *reinterpret_cast<const f32x4 *>(now + r16 * P + STEPS * g + 4 * i);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = now[r16 * P + 4 * (4 * i + e) + g];
#pragma unroll
            for (int e = 0; e < 4; ++e) n[e & 1] = mfma4(x[e], m[i][e], n[e & 1]);
        }
        s = n[0] + n[1];
        const int next = BACK ? seg - 1 : seg + 1;
        ask(min(max(next, 0), a.segments - 1));
    }
}

template <typename T, int DK, bool FULL> void scan(const GDelta &a, int what, bool ends, dim3 grid, hipStream_t stream)
{
    if (what == kForward) {
        scan_kernel<T, DK, FULL, kForward><<<grid, 512, 0, stream>>>(a);
    } else if (what == kKeep) {
        scan_kernel<T, DK, FULL, kKeep><<<grid, 512, 0, stream>>>(a);
    } else if (what == kEnds) {
        scan_kernel<T, DK, FULL, kEnds><<<grid, 512, 0, stream>>>(a);
    } else {
        // Backward: a third group of wavefronts where every workgroup has a compute unit for itself (2 x 8192 tokens, 16 heads of 128: 383 ->
        // 373 us; d_k up to 64: of three groups no two workgroups have their registers there.  Of 128 none have their LDS anyway, 103 KB, and with more
        // workgroups than compute units three groups are faster as well: the whole backward of 4 x 4096 tokens of 16 heads 1148 -> 1062 us.  That is not taken yet).
        // Wider or fp32: their values do not fit a third group's.
        if constexpr (sizeof(T) == 2 && DK <= 128)
            if (grid.x <= (unsigned)device_cu_count()) {
                scan_bwd_kernel<T, DK, FULL, 3><<<grid, 768, 0, stream>>>(a, ends);
                return;
            }
        scan_bwd_kernel<T, DK, FULL, 2><<<grid, 512, 0, stream>>>(a, ends);
    }
}
template <typename T, int DK> hipError_t scan(const GDelta &a, int what, hipStream_t stream)
{
    const bool full = gdelta_full(a, sizeof(T));
    const int wide = (a.dv + 31) / 32 * 32;
    auto run = [&](int how, bool ends) {
        const int rows = how == kForward ? a.dv : how == kEnds ? wide + DK : wide;
        const dim3 grid((unsigned)((long long)a.N * a.Hv * a.segments * ((rows + N - 1) / N)));
        full ? scan<T, DK, true>(a, how, ends, grid, stream) : scan<T, DK, false>(a, how, ends, grid, stream);
        return hipGetLastError();
    };
    if (a.segments > 1) {
        const dim3 grid((unsigned)((long long)a.N * a.Hv * (wide / N)));
        if (hipError_t e = run(what == kBackward ? kBackward : kEnds, what == kBackward)) return e;
        what == kBackward ? join_kernel<DK, true><<<grid, 4 * DK, 0, stream>>>(a) : join_kernel<DK, false><<<grid, 4 * DK, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return run(what, false);
}
template <typename T> hipError_t scan(const GDelta &a, int what, hipStream_t stream)
{
    return a.dk <= 64 ? scan<T, 64>(a, what, stream) : a.dk <= 128 ? scan<T, 128>(a, what, stream) : scan<T, 256>(a, what, stream);
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
