// Gated delta rule (include/pf_layer.h): what its kernels share.  Per sequence and value head, with a_t = exp(g_t),
//
//   S_t = a_t S_{t-1} (I - beta_t k_t k_t^T) + beta_t v_t k_t^T ,   o_t = S_t q_t .
//
// In a chunk of 64 tokens with G_i = g_1 + .. + g_i, D_ij = exp(G_i - G_j), gamma_i = exp(G_i), delta_i = exp(G_64 - G_i) and the state
// S before it,
//
//   T = (I + A)^-1 ,  A_ij = beta_i D_ij k_i.k_j (j < i) ,  P_ij = D_ij q_i.k_j (j <= i)      each chunk by itself: the flow kernel
//   U = T beta (V - gamma K S^T) ,  O = gamma Q S^T + P U ,  S' = gamma_64 S + (delta U)^T K  chunk after chunk: the scan kernel
//
// Numbers.  The state and everything that it is made from are held in fp32 and multiplied as such.  An fp32 matrix instruction does 64
// operations a cycle, the bf16 one 1024, so numbers are split into bf16 ones whose sum they are: three of them (24 bits) on the way into a
// state, two (16 bits) on the way into an output that is rounded to bf16.  (Three there too, 0.02 % of the bf16 outputs in the place of 0.36 % are rounded other
// than those of 24 bits are, with the same error against exact ones, 1.65e-3; but a second workgroup's LDS is gone: 4 x 4096 tokens of 16 heads of 128
// take 314 us, not 244, 65536 of 32 heads 2627, not 2430.)  An input in bf16 is one part by itself: three products of
// 32 steps take 48 cycles where the fp32 instructions take 256; of three parts times three the six products down to 2^-24, 96
// cycles.  Inputs in fp32 take the fp32 instruction.
#pragma once
#include "pf_layer_common.h"
#include "pf_layer_internal.h"

namespace pf {
namespace gd {

constexpr int C = kGDeltaChunk;      // tokens of a chunk

// ---- fragments of the 16x16x32 product: eight consecutive steps 8 g .. 8 g + 7 of row (column) r16
template <typename T> struct In;               // of an input, exact
template <> struct In<bf16> { bf16x8 v; };
template <> struct In<float> { f32x8 v; };
template <typename T, int NP> struct Of;       // of a number computed here: its NP parts, the largest first, or itself
template <int NP> struct Of<bf16, NP> { bf16x8 p[NP]; };
template <int NP> struct Of<float, NP> { f32x8 v; };

__device__ __forceinline__ f32x4 mma8(f32x8 a, f32x8 b, f32x4 c)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) c = mfma4(a[e], b[e], c);
    return c;
}
// 16 steps, 4 g .. 4 g + 3 of a lane, in fp32
__device__ __forceinline__ f32x4 mma4(f32x4 a, f32x4 b, f32x4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = mfma4(a[e], b[e], c);
    return c;
}
__device__ __forceinline__ f32x4 mma(In<bf16> a, In<bf16> b, f32x4 c) { return mfma16(a.v, b.v, c); }
__device__ __forceinline__ f32x4 mma(In<float> a, In<float> b, f32x4 c) { return mma8(a.v, b.v, c); }
// USE: how many of b's parts
template <int USE, int NP> __device__ __forceinline__ f32x4 mma(In<bf16> a, const Of<bf16, NP> &b, f32x4 c)
{
#pragma unroll
    for (int p = USE - 1; p >= 0; --p) c = mfma16(a.v, b.p[p], c);
    return c;
}
template <int USE, int NP> __device__ __forceinline__ f32x4 mma(In<float> a, const Of<float, NP> &b, f32x4 c) { return mma8(a.v, b.v, c); }
template <int USE, int NP, typename T> __device__ __forceinline__ f32x4 mma(const Of<T, NP> &a, In<T> b, f32x4 c)
{
    if constexpr (sizeof(T) == 4) {
        return mma8(a.v, b.v, c);
    } else {
#pragma unroll
        for (int p = USE - 1; p >= 0; --p) c = mfma16(a.p[p], b.v, c);
        return c;
    }
}
// N results side by side, c += a b for one b: a product that adds to the result of the one before it waits for that
template <typename T, int N> __device__ __forceinline__ void mma_each(const In<T> (&a)[N], const Of<T, 3> &b, f32x4 (&c)[N])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < N; ++i) c[i] = mfma4(a[i].v[e], b.v[e], c[i]);
    } else {
#pragma unroll
        for (int p = 2; p >= 0; --p)
#pragma unroll
            for (int i = 0; i < N; ++i) c[i] = mfma16(a[i].v, b.p[p], c[i]);
    }
}
// two computed numbers of two parts each: the product of the small parts is left out (2^-18)
template <typename T> __device__ __forceinline__ f32x4 mma22(const Of<T, 2> &a, const Of<T, 2> &b, f32x4 c)
{
    if constexpr (sizeof(T) == 4) {
        return mma8(a.v, b.v, c);
    } else {
        c = mfma16(a.p[1], b.p[0], c);
        c = mfma16(a.p[0], b.p[1], c);
        return mfma16(a.p[0], b.p[0], c);
    }
}

__device__ __forceinline__ f32x8 stack(f32x4 a, f32x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
// three parts each: what is left out is 2^-24 of the whole
__device__ __forceinline__ f32x4 mma33(const Of<bf16, 3> &a, const Of<bf16, 3> &b, f32x4 c)
{
    c = mfma16(a.p[2], b.p[0], c);
    c = mfma16(a.p[1], b.p[1], c);
    c = mfma16(a.p[0], b.p[2], c);
    c = mfma16(a.p[1], b.p[0], c);
    c = mfma16(a.p[0], b.p[1], c);
    return mfma16(a.p[0], b.p[0], c);
}
template <int NP> __device__ __forceinline__ f32x4 mma_parts(const Of<bf16, NP> &a, const Of<bf16, NP> &b, f32x4 c)
{
    if constexpr (NP == 2) return mma22<bf16>(a, b, c);
    else return mma33(a, b, c);
}

template <int N> struct F32s;
template <> struct F32s<4> { typedef f32x4 f; typedef bf16x4 b; };
template <> struct F32s<8> { typedef f32x8 f; typedef bf16x8 b; };
// x as a sum of NP bf16 numbers, each the rest rounded to nearest even (two at a time: a pair of conversions is one instruction)
template <int NP, int N> __device__ __forceinline__ void split(typename F32s<N>::f x, typename F32s<N>::b (&p)[NP])
{
    uint32_t r[NP][N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
        f32x2 v = {x[2 * j], x[2 * j + 1]};
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const uint32_t u = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
            r[i][j] = u;
            if (i + 1 < NP) v[0] -= __uint_as_float(u << 16), v[1] -= __uint_as_float(u & 0xffff0000u);
        }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) __builtin_memcpy(&p[i], r[i], sizeof(p[i]));
}
// parts times an input; one in fp32 is split as well
__device__ __forceinline__ f32x4 mma_input(const Of<bf16, 3> &a, In<bf16> b, f32x4 c) { return mma<3>(a, b, c); }
__device__ __forceinline__ f32x4 mma_input(const Of<bf16, 3> &a, In<float> b, f32x4 c)
{
    Of<bf16, 3> p;
    split<3, 8>(b.v, p.p);
    return mma33(a, p, c);
}
template <typename T, int NP> __device__ __forceinline__ Of<T, NP> of(f32x8 x)
{
    Of<T, NP> r;
    if constexpr (sizeof(T) == 4) r.v = x;
    else split<NP, 8>(x, r.p);
    return r;
}
__device__ __forceinline__ f32x8 in_f32(In<float> a) { return a.v; }
__device__ __forceinline__ f32x8 in_f32(In<bf16> a) { return __builtin_convertvector(a.v, f32x8); }

// ---- tiles in LDS
// Inputs: rows of K elements, 16 bytes of padding, so that the rows that 16 lanes read lie four banks apart.
template <typename T> constexpr int pitch(int K) { return K + 16 / (int)sizeof(T); }

template <typename T> __device__ __forceinline__ In<T> frag_rows(const T *tile, int ld, int row, int k)
{
    In<T> r;
    __builtin_memcpy(&r, __builtin_assume_aligned(tile + row * ld + k, 16), sizeof(r));
    return r;
}
// steps k .. along the tile's rows, column n: k the lane's 8 g, n the 16 lanes' first
template <typename T> __device__ __forceinline__ In<T> frag_cols(const T *tile, int ld, int k, int n, int r16)
{
    In<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = tile[(k + e) * ld + n + r16];
    } else {
        const T *p = tile + (k + (r16 >> 2)) * ld + n + 4 * (r16 & 3);
        r.v = join(lds_read_tr4(p), lds_read_tr4(p + 4 * ld));
    }
    return r;
}

// the same, but the 16 lanes have the columns n + 8 (r16 / 4) + 4 half + r16 % 4: of two such fragments' results, half = 0 and 1, a lane
// has the eight neighbours n + 8 g ..
template <typename T> __device__ __forceinline__ In<T> frag_cols8(const T *tile, int ld, int k, int n, int half, int r16)
{
    In<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = tile[(k + e) * ld + n + 8 * (r16 >> 2) + 4 * half + (r16 & 3)];
    } else {
        const T *p = tile + (k + (r16 >> 2)) * ld + n + 8 * (r16 & 3) + 4 * half;
        r.v = join(lds_read_tr4(p), lds_read_tr4(p + 4 * ld));
    }
    return r;
}

// Computed numbers, R rows of K: NP planes of bf16, or fp32.
template <typename T, int NP, int R, int K> struct Tile {
    static constexpr int kLd = pitch<T>(K), kPlane = R * kLd, kBytes = (sizeof(T) == 4 ? 1 : NP) * kPlane * (int)sizeof(T);
    T *at;
    __device__ __forceinline__ void put4(int row, int k, f32x4 x) const      // k: a multiple of 4
    {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4 *>(at + row * kLd + k) = x;
        } else {
            bf16x4 p[NP];
            split<NP, 4>(x, p);
#pragma unroll
            for (int i = 0; i < NP; ++i) *reinterpret_cast<bf16x4 *>(at + i * kPlane + row * kLd + k) = p[i];
        }
    }
    // the first parts of eight neighbours
    template <int PARTS> __device__ __forceinline__ void put8(int row, int k, const Of<T, PARTS> &x) const
    {
        static_assert(NP <= PARTS);
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4 *>(at + row * kLd + k) = __builtin_shufflevector(x.v, x.v, 0, 1, 2, 3);
            *reinterpret_cast<f32x4 *>(at + row * kLd + k + 4) = __builtin_shufflevector(x.v, x.v, 4, 5, 6, 7);
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) st8(at + i * kPlane + row * kLd + k, x.p[i]);
        }
    }
    __device__ __forceinline__ Of<T, NP> rows(int row, int k) const
    {
        Of<T, NP> r;
        if constexpr (sizeof(T) == 4) r.v = frag_rows(at, kLd, row, k).v;
        else
#pragma unroll
            for (int i = 0; i < NP; ++i) r.p[i] = frag_rows(at + i * kPlane, kLd, row, k).v;
        return r;
    }
    __device__ __forceinline__ Of<T, NP> cols(int k, int n, int r16) const
    {
        Of<T, NP> r;
        if constexpr (sizeof(T) == 4) r.v = frag_cols(at, kLd, k, n, r16).v;
        else
#pragma unroll
            for (int i = 0; i < NP; ++i) r.p[i] = frag_cols(at + i * kPlane, kLd, k, n, r16).v;
        return r;
    }
};

// ---- inputs in memory
// Eight of a row's values from its k-th on, `left` of them (FULL: eight, at a multiple of 16 bytes); zeros in the place of the others.
template <typename T, bool FULL> __device__ __forceinline__ In<T> fetch(const T *p, int left)
{
    return __builtin_bit_cast(In<T>, load8<T, FULL>(p, FULL ? 8 : left));
}

// ---- chunks
struct Chunk {
    int seq, c, tok, len;      // sequence, chunk in it, its first token's row among the rows of the sequence's batch, tokens (1 .. 64)
};
// Packed sequences: where each starts, its length, its first chunk; and of each chunk its sequence (-1: there is none).
struct Plan {
    int *start, *len, *first, *of;
};
__host__ __device__ inline Plan plan_of(int *p, int N) { return {p, p + N, p + 2 * N, p + 3 * N}; }

// (what is the same for a whole wavefront, in scalar registers: addresses that come from it cost the vector unit nothing)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ bool chunk_at(const GDelta &a, int id, Chunk &x)
{
    if (a.offsets) {
        const Plan p = plan_of(a.plan, a.N);
        x.seq = uniform(p.of[id]);
        if (x.seq < 0) return false;
        x.c = id - uniform(p.first[x.seq]);
        x.tok = uniform(p.start[x.seq]) + C * x.c;
        x.len = min(C, uniform(p.len[x.seq]) - C * x.c);
    } else {
        x.seq = id / a.per;
        x.c = id - x.seq * a.per;
        x.tok = C * x.c;
        x.len = min(C, a.L - x.tok);
    }
    return true;
}
struct Sequence {
    int tok, len, first;      // its first token's row, tokens, first chunk
};
__device__ __forceinline__ Sequence sequence_at(const GDelta &a, int seq)
{
    if (a.offsets) {
        if (a.chunks == 0) return {0, 0, 0};
        const Plan p = plan_of(a.plan, a.N);
        return {uniform(p.start[seq]), uniform(p.len[seq]), uniform(p.first[seq])};
    }
    return {0, a.L, seq * a.per};
}
// row of the dense outputs [.., tokens, H, d]
__device__ __forceinline__ long long out_row(const GDelta &a, int seq, int tok) { return (long long)seq * a.rows + tok; }

// ---- what the flow kernel leaves for each chunk and value head.  Matrices of pairs of tokens, as three bf16 numbers each (24 bits): T and
// P (of P as many as the forward uses), for the backward T and the transposes of both.  They are kept as the fragments that the
// scans take, 16 rows by 32 columns, each part of one 1 KB as its 64 lanes hold it, and of the triangle only: rows 16 w .. have the
// columns up to theirs (transposed: from theirs on), six fragments.
constexpr int kMatrix = 6 * 3 * 512;
__host__ __device__ constexpr int low_fragment(int w, int t) { return w < 2 ? w : 2 * w - 2 + t; }
__host__ __device__ constexpr int high_fragment(int w, int t) { return w < 2 ? 2 * w + t : w + 2; }
// and of each token: gamma, delta, beta, and G in units of log 2 as two numbers, a multiple of 1/16 and the rest, so that differences
// of far sums keep their last bits
constexpr int kVec = 5 * C;
struct Vec {
    const float *gamma, *delta, *beta, *coarse, *fine;
};
__device__ __forceinline__ Vec vec_at(const float *vec, long long x)
{
    const float *p = vec + x * kVec;
    return {p, p + C, p + 2 * C, p + 3 * C, p + 4 * C};
}
// 2^(coarse + fine), coarse a multiple of 1/16
__device__ __forceinline__ float power(float coarse, float fine)
{
    const float n = __builtin_rintf(coarse);
    return __builtin_ldexpf(__builtin_amdgcn_exp2f((coarse - n) + fine), (int)n);
}
__device__ __forceinline__ float coarse_of(double x) { return (float)(__builtin_rint(x * 16.) * 0.0625); }
__device__ __forceinline__ float power(double x)
{
    const float coarse = coarse_of(x);
    return power(coarse, (float)(x - coarse));
}

// The log of a gate as it is used: exp(-256) and exp(256) are 0 and infinite in fp32, also times what else it holds beside them here.
__device__ __forceinline__ float gate_in(float g) { return g < -256.f ? -256.f : g > 256.f ? 256.f : g; }
constexpr double kLog2e = 1.4426950408889634;

__device__ __forceinline__ f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ float to_f32(bf16 x) { return (float)x; }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// S += (two lanes apart by 16, 32): over the four groups of 16 lanes
__device__ __forceinline__ float sum_of_groups(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

}  // namespace gd
}  // namespace pf
