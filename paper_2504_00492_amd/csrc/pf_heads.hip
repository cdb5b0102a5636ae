// Norm of every head of queries and keys with the rotation by the token's position, and its backward (include/pf_layer.h).  Memory
// is what bounds both: a row is read once and written once (the backward reads two).
//
// A row of d values is cut into units of eight for a lane: the turned ones four pairs at a time, a and b of a pair in the same lane (in
// halves they lie rot / 2 apart, else side by side), the others as they follow.  A wavefront has the rows of one token, 64 / LPR of them
// side by side, and its cosines and sines are read once for all heads that it takes.
#include "pf_layer_common.h"
#include "pf_layer_internal.h"

namespace pf {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

// over LPR neighbouring lanes
template <int LPR> __device__ __forceinline__ float row_sum(float s)
{
    auto dpp = [](float v, auto ctrl) {
        return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    if constexpr (LPR == 8) {
        s += dpp(s, std::integral_constant<int, 0xb1>{});       // quad_perm 1 0 3 2
        s += dpp(s, std::integral_constant<int, 0x4e>{});       // quad_perm 2 3 0 1
        return s + dpp(s, std::integral_constant<int, 0x141>{});      // row_half_mirror
    } else {
        s = sum_of_16(s);
        if constexpr (LPR >= 32) s += __shfl_xor(s, 16);
        if constexpr (LPR >= 64) s += __shfl_xor(s, 32);
        return s;
    }
}

struct Unit {
    int p0, p1, n0, n1, pair;      // two pieces of up to four values; the first pair's number, or -1
};
__device__ __forceinline__ Unit unit_at(const Heads &a, int u)
{
    const int half = a.rot / 2, turning = (half + 3) / 4;
    Unit x;
    if (u < turning) {
        const int n = min(4, half - 4 * u);      // pairs
        x.pair = 4 * u;
        x.p0 = a.pairs ? 8 * u : 4 * u;
        x.p1 = a.pairs ? 8 * u + 4 : half + 4 * u;
        x.n0 = a.pairs ? min(4, 2 * n) : n;
        x.n1 = a.pairs ? 2 * n - x.n0 : n;
    } else {
        x.pair = -1;
        x.p0 = a.rot + 8 * (u - turning), x.p1 = x.p0 + 4;
        x.n0 = min(4, max(0, a.d - x.p0)), x.n1 = min(4, max(0, a.d - x.p1));
    }
    return x;
}

// Four values of which n are there.  FAST: none or four, at a multiple of their size.
template <typename T, bool FAST> __device__ __forceinline__ f4 get(const T *p, int n)
{
    typedef T t4 __attribute__((ext_vector_type(4)));
    f4 r = {0.f, 0.f, 0.f, 0.f};
    if constexpr (FAST) {
        if (n) r = __builtin_convertvector(*reinterpret_cast<const t4 *>(p), f4);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) r[e] = (float)p[e];
    }
    return r;
}
template <typename T, bool FAST> __device__ __forceinline__ void set(T *p, int n, f4 v)
{
    typedef T t4 __attribute__((ext_vector_type(4)));
    if constexpr (FAST) {
        if (n) *reinterpret_cast<t4 *>(p) = __builtin_convertvector(v, t4);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) p[e] = (T)v[e];
    }
}
// first and second values of four pairs out of the two pieces, and back
__device__ __forceinline__ void apart(bool pairs, f4 &x, f4 &y)
{
    if (!pairs) return;
    const f4 a = {x[0], x[2], y[0], y[2]}, b = {x[1], x[3], y[1], y[3]};
    x = a, y = b;
}
__device__ __forceinline__ void together(bool pairs, f4 &x, f4 &y)
{
    if (!pairs) return;
    const f4 a = {x[0], y[0], x[1], y[1]}, b = {x[2], y[2], x[3], y[3]};
    x = a, y = b;
}
// cosines and sines of a unit's pairs at a position of the table (NaN where there is no such position)
template <bool FAST> __device__ __forceinline__ void turns(const Heads &a, const Unit &x, int token, f4 &c, f4 &s)
{
    c = {1.f, 1.f, 1.f, 1.f}, s = {0.f, 0.f, 0.f, 0.f};
    if (x.pair < 0) return;
    const int at = a.positions[token];
    if (at < 0 || at >= a.far) {
        c = s = __builtin_nanf("") + c;
        return;
    }
    const float *row = a.table + (long long)at * a.rot + x.pair;
    const int n = min(4, a.rot / 2 - x.pair);
    c = get<float, FAST>(row, n), s = get<float, FAST>(row + a.rot / 2, n);
}

constexpr int kAhead = 4;      // rows of a lane under way together

template <typename T, int LPR, bool FAST>
__global__ __launch_bounds__(256) void heads_fwd_kernel(Heads a, int groups, int each)
{
    constexpr int ROWS = 64 / LPR;
    const int wave = (int)((blockIdx.x * 256ll + threadIdx.x) >> 6), lane = threadIdx.x & 63;
    const int token = wave / groups, first = (wave - token * groups) * each;
    if (token >= a.M) return;
    const int H0 = a.side[0].H, H = H0 + a.side[1].H, end = min(H, first + each);
    const Unit x = unit_at(a, lane % LPR);
    f4 c, s, w[2][2];
    turns<FAST>(a, x, token, c, s);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const T *p = static_cast<const T *>(a.side[i].w);
        w[i][0] = w[i][1] = f4{1.f, 1.f, 1.f, 1.f};
        if (p) w[i][0] = get<T, FAST>(p + x.p0, x.n0), w[i][1] = get<T, FAST>(p + x.p1, x.n1);
        w[i][0] *= a.side[i].scale, w[i][1] *= a.side[i].scale;
        apart(a.pairs, w[i][0], w[i][1]);
    }
    const float share = a.l2 ? 1.f : 1.f / (float)a.d;
    for (int h0 = first + lane / LPR; h0 < end; h0 += ROWS * kAhead) {
        f4 u[kAhead], v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = h0 + i * ROWS;
            u[i] = v[i] = f4{0.f, 0.f, 0.f, 0.f};
            if (h < end) {
                const bool k = h >= H0;
                const T *p = static_cast<const T *>(k ? a.side[1].X : a.side[0].X) + token * (k ? a.side[1].xt : a.side[0].xt) +
                             (k ? h - H0 : h) * (k ? a.side[1].xh : a.side[0].xh);
                u[i] = get<T, FAST>(p + x.p0, x.n0), v[i] = get<T, FAST>(p + x.p1, x.n1);
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = h0 + i * ROWS;
            float squares = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) squares += u[i][e] * u[i][e] + v[i][e] * v[i][e];
            const float rho = 1.f / sqrtf(row_sum<LPR>(squares) * share + a.eps);
            if (h >= end) continue;
            const bool k = h >= H0;
            apart(a.pairs, u[i], v[i]);
            const f4 p = u[i] * rho * (k ? w[1][0] : w[0][0]), q = v[i] * rho * (k ? w[1][1] : w[0][1]);
            f4 y = p * c - q * s, z = p * s + q * c;
            together(a.pairs, y, z);
            T *to = static_cast<T *>(k ? a.side[1].Y : a.side[0].Y) + ((long long)token * (k ? H - H0 : H0) + (k ? h - H0 : h)) * a.d;
            set<T, FAST>(to + x.p0, x.n0, y), set<T, FAST>(to + x.p1, x.n1, z);
        }
    }
}

// With n the norm's divisor, xh = x / n and g = w times the gradient turned back: dx = (g - xh (mean or sum of g xh)) / n, dw the sum of
// the gradient turned back times xh; these sums stay with a lane over all rows of its wavefront, then one part for each workgroup.
template <typename T, int LPR, bool FAST, bool WEIGHTS>
__global__ __launch_bounds__(256) void heads_bwd_kernel(Heads a, int groups, int each)
{
    constexpr int ROWS = 64 / LPR, AHEAD = 2;
    const int lane = threadIdx.x & 63, waves = (int)gridDim.x * 4;
    const int H0 = a.side[0].H, H = H0 + a.side[1].H;
    const Unit x = unit_at(a, lane % LPR);
    f4 w[2][2], dw[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const T *p = static_cast<const T *>(a.side[i].w);
        w[i][0] = w[i][1] = f4{1.f, 1.f, 1.f, 1.f};
        if (p) w[i][0] = get<T, FAST>(p + x.p0, x.n0), w[i][1] = get<T, FAST>(p + x.p1, x.n1);
        apart(a.pairs, w[i][0], w[i][1]);
        dw[i][0] = dw[i][1] = f4{0.f, 0.f, 0.f, 0.f};
    }
    const float share = a.l2 ? 1.f : 1.f / (float)a.d;
    const long long items = (long long)a.M * groups;
    for (long long item = (blockIdx.x * 256ll + threadIdx.x) >> 6; item < items; item += waves) {
        const int token = (int)(item / groups), first = (int)(item - (long long)token * groups) * each, end = min(H, first + each);
        f4 c, s;
        turns<FAST>(a, x, token, c, s);
        for (int h0 = first + lane / LPR; h0 < end; h0 += ROWS * AHEAD) {
            f4 u[AHEAD], v[AHEAD], p[AHEAD], q[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int h = h0 + i * ROWS;
                u[i] = v[i] = p[i] = q[i] = f4{0.f, 0.f, 0.f, 0.f};
                if (h < end) {
                    const bool k = h >= H0;
                    const HeadSide &o = a.side[0], &t = a.side[1];
                    const int hh = k ? h - H0 : h;
                    const T *from = static_cast<const T *>(k ? t.X : o.X) + token * (k ? t.xt : o.xt) + hh * (k ? t.xh : o.xh);
                    const T *grad = static_cast<const T *>(k ? t.dY : o.dY) + token * (k ? t.dyt : o.dyt) + hh * (k ? t.dyh : o.dyh);
                    u[i] = get<T, FAST>(from + x.p0, x.n0), v[i] = get<T, FAST>(from + x.p1, x.n1);
                    p[i] = get<T, FAST>(grad + x.p0, x.n0), q[i] = get<T, FAST>(grad + x.p1, x.n1);
                }
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int h = h0 + i * ROWS;
                const bool k = h >= H0;
                float squares = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) squares += u[i][e] * u[i][e] + v[i][e] * v[i][e];
                const float rho = 1.f / sqrtf(row_sum<LPR>(squares) * share + a.eps), scale = k ? a.side[1].scale : a.side[0].scale;
                apart(a.pairs, u[i], v[i]);
                apart(a.pairs, p[i], q[i]);
                u[i] *= rho, v[i] *= rho;
                const f4 back = scale * (p[i] * c + q[i] * s), next = scale * (q[i] * c - p[i] * s);
                const f4 g = back * (k ? w[1][0] : w[0][0]), f = next * (k ? w[1][1] : w[0][1]);
                float along = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) along += g[e] * u[i][e] + f[e] * v[i][e];
                along = row_sum<LPR>(along) * share;
                if (h >= end) continue;
                if constexpr (WEIGHTS) {
                    const f4 m = back * u[i], n = next * v[i], none = {0.f, 0.f, 0.f, 0.f};
                    dw[0][0] += k ? none : m, dw[0][1] += k ? none : n;
                    dw[1][0] += k ? m : none, dw[1][1] += k ? n : none;
                }
                f4 y = rho * (g - u[i] * along), z = rho * (f - v[i] * along);
                together(a.pairs, y, z);
                T *to = static_cast<T *>(k ? a.side[1].Y : a.side[0].Y) + ((long long)token * (k ? H - H0 : H0) + (k ? h - H0 : h)) * a.d;
                set<T, FAST>(to + x.p0, x.n0, y), set<T, FAST>(to + x.p1, x.n1, z);
            }
        }
    }
    if constexpr (WEIGHTS) {
        __shared__ f4 sums[4][64][2];
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i) __syncthreads();
            sums[wave][lane][0] = dw[i][0], sums[wave][lane][1] = dw[i][1];
            __syncthreads();
            if (threadIdx.x < LPR) {      // (a unit's lanes of all rows and wavefronts, in their order)
                f4 u = {0.f, 0.f, 0.f, 0.f}, v = u;
                for (int r = 0; r < 4 * ROWS; ++r) {
                    u += sums[r / ROWS][r % ROWS * LPR + lane][0], v += sums[r / ROWS][r % ROWS * LPR + lane][1];
                }
                together(a.pairs, u, v);
                float *to = a.part + ((long long)i * gridDim.x + blockIdx.x) * a.d;
                set<float, false>(to + x.p0, x.n0, u), set<float, false>(to + x.p1, x.n1, v);
            }
        }
    }
}

// dw out of the workgroups' parts: 16 columns to a workgroup, 16 threads to a column
__global__ __launch_bounds__(256) void heads_sum_kernel(Heads a, int parts)
{
    __shared__ float sums[16][17];
    const int side = blockIdx.y, col = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4;
    float *dw = a.side[side].dw;
    float sum = 0.f;
    if (dw && col < a.d) {
        const float *p = a.part + (long long)side * parts * a.d + col;
        int i = r;
        for (; i + 7 * 16 < parts; i += 8 * 16) {      // (eight loads under way together)
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p[(long long)(i + 16 * j) * a.d];
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += v[j];
        }
        for (; i < parts; i += 16) sum += p[(long long)i * a.d];
    }
    sums[r][threadIdx.x & 15] = sum;
    __syncthreads();
    if (r == 0 && dw && col < a.d) {
        float all = 0.f;
        for (int i = 0; i < 16; ++i) all += sums[i][threadIdx.x];
        dw[col] = all;
    }
}

// heads that a wavefront takes one after another, so that there are enough wavefronts, and how many such groups a token has
struct Share {
    int each, groups;
};
Share share_of(int M, int H, int rows)
{
    int each = rows;
    while (each < H && (double)M * ((H + 2 * each - 1) / (2 * each)) >= 8192) each *= 2;
    return {each, (H + each - 1) / each};
}
int lanes_of(int units) { return units <= 8 ? 8 : units <= 16 ? 16 : units <= 32 ? 32 : 64; }

bool fast(const Heads &a, int size, bool backward)
{
    uintptr_t all = 0;
    long long strides = 0;
    for (const HeadSide &s : a.side) {
        if (!s.H) continue;
        all |= reinterpret_cast<uintptr_t>(s.X), strides |= s.xt | s.xh;
        if (backward) all |= reinterpret_cast<uintptr_t>(s.dY), strides |= s.dyt | s.dyh;
    }
    return a.d % 4 == 0 && a.rot % 8 == 0 && (all | (uintptr_t)(strides * size)) % (4 * size) == 0;
}

template <typename T, int LPR> hipError_t forward(const Heads &a, hipStream_t stream)
{
    const Share x = share_of(a.M, a.side[0].H + a.side[1].H, 64 / LPR);
    const double groups = ((double)a.M * x.groups + 3) / 4;
    if (!launch_holds(groups, 256)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)groups);
    if (fast(a, sizeof(T), false)) heads_fwd_kernel<T, LPR, true><<<grid, 256, 0, stream>>>(a, x.groups, x.each);
    else heads_fwd_kernel<T, LPR, false><<<grid, 256, 0, stream>>>(a, x.groups, x.each);
    return hipGetLastError();
}
template <typename T, int LPR> hipError_t backward(const Heads &a, hipStream_t stream)
{
    const Share x = share_of(a.M, a.side[0].H + a.side[1].H, 64 / LPR);
    const int parts = heads_bwd_parts(a.M, a.side[0].H, a.side[1].H, a.d, a.rot);
    const bool f = fast(a, sizeof(T), true), weights = a.side[0].dw || a.side[1].dw;
    if (parts == 0)      // (no rows: dw are zeros)
        ;
    else if (f)
        weights ? heads_bwd_kernel<T, LPR, true, true><<<parts, 256, 0, stream>>>(a, x.groups, x.each)
                : heads_bwd_kernel<T, LPR, true, false><<<parts, 256, 0, stream>>>(a, x.groups, x.each);
    else
        weights ? heads_bwd_kernel<T, LPR, false, true><<<parts, 256, 0, stream>>>(a, x.groups, x.each)
                : heads_bwd_kernel<T, LPR, false, false><<<parts, 256, 0, stream>>>(a, x.groups, x.each);
    if (hipError_t e = hipGetLastError()) return e;
    if (weights) heads_sum_kernel<<<dim3((a.d + 15) / 16, 2), 256, 0, stream>>>(a, parts);
    return hipGetLastError();
}
template <typename T> hipError_t heads(const Heads &a, bool back, hipStream_t stream)
{
    switch (lanes_of(head_units(a.d, a.rot))) {
    case 8: return back ? backward<T, 8>(a, stream) : forward<T, 8>(a, stream);
    case 16: return back ? backward<T, 16>(a, stream) : forward<T, 16>(a, stream);
    case 32: return back ? backward<T, 32>(a, stream) : forward<T, 32>(a, stream);
    default: return back ? backward<T, 64>(a, stream) : forward<T, 64>(a, stream);
    }
}

}  // namespace

// workgroups of the backward: as many as fill the chip twice over, and no more than there is work for
int heads_bwd_parts(int M, int Hq, int Hk, int d, int rot)
{
    const int rows = 64 / lanes_of(head_units(d, rot));
    const double groups = ((double)M * share_of(M, Hq + Hk, rows).groups + 3) / 4;
    return groups < 2048 ? (int)groups : 2048;
}
hipError_t launch_heads_fwd(const Heads &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? heads<bf16>(a, false, stream) : heads<float>(a, false, stream);
}
hipError_t launch_heads_bwd(const Heads &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? heads<bf16>(a, true, stream) : heads<float>(a, true, stream);
}

}  // namespace pf
