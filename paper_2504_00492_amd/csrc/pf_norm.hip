// Root-mean-square norm of rows with the residual's addition before it and an output in 8 bits, and its backward.
//
// A row is held in registers by G lanes, eight consecutive values a lane and step (NV steps), so that memory sees every
// array once: x, r and what is written, nothing else.  Sixteen lanes then hold 128 columns, the block of one scale.  G goes by
// the width alone: up to 128 columns a row to 16 lanes, four rows to a wavefront, and no barrier up to 1024 columns.
//
// Bound by HBM (a plain copy reaches 5.1 TB/s): forward 32768 x 4096, residual in, sum and 8 bits out, bf16, 174 us, 5.4 TB/s; 262144 x 128 into
// bf16 21.2 us, 6.3; backward 8191 x 4096 48.5 us and 4.1 for the sums of dw, 5.0 TB/s; a few rows: 3.8 us, what a launch takes.
#include "pf_layer_common.h"
#include "pf_layer_internal.h"

#include <type_traits>

namespace pf {

namespace {

// Sum over the G lanes of a row; all of them get it, summed in the same order.  G > 64: `part` (two sets in turn, so that
// one barrier a call is enough) carries the wavefronts' sums.
template <int G, int N> struct RowSum {
    float (*part)[N][16];
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&s)[N])
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            s[n] = sum_of_16(s[n]);
            if constexpr (G >= 64) {
                s[n] += __shfl_xor(s[n], 16);
                s[n] += __shfl_xor(s[n], 32);
            }
        }
        if constexpr (G > 64) {
            const int w = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int n = 0; n < N; ++n) part[turn][n][w] = s[n];
            __syncthreads();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                s[n] = part[turn][n][0];
#pragma unroll
                for (int i = 1; i < G / 64; ++i) s[n] += part[turn][n][i];
            }
            turn ^= 1;
        }
    }
};

template <int G> constexpr int kThreads = G < 256 ? 256 : G;

// 1 / sqrt(mean + eps), to the last bit or so: the instruction's one is off by up to one unit more
__device__ __forceinline__ float inverse_root(float x) { return 1.f / sqrtf(x); }

template <typename T, bool VEC, int G, int NV>
__global__ __launch_bounds__(kThreads<G>) void norm_fwd_kernel(NormFwd a)
{
    constexpr int rows = kThreads<G> / G;
    __shared__ float part[2][1][16];
    RowSum<G, 1> sum{part};
    const int lane = threadIdx.x % G;
    const T *X = static_cast<const T *>(a.X), *R = static_cast<const T *>(a.R);
    auto col = [&](int i) { return (i * G + lane) * 8; };
    Raw8<T, VEC> w[NV];
    if (a.w)
#pragma unroll
        for (int i = 0; i < NV; ++i) w[i] = load8<T, VEC>(static_cast<const T *>(a.w) + col(i), a.D - col(i));
    // 16 neighbouring rows on one XCD: a block's scales of neighbouring rows lie side by side, and meet in its L2 (32768 rows of 4096:
    // 407 MB written instead of 441; all of an XCD's rows side by side write as little, but 189 us instead of 176)
    const unsigned b = blockIdx.x, first = (b | 127) < gridDim.x ? (b & ~127u) | (b & 7) << 4 | (b >> 3 & 15) : b;
    for (long long row = (long long)first * rows + threadIdx.x / G; row < a.M; row += (long long)gridDim.x * rows) {
        Raw8<T, VEC> x[NV], r[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = load8<T, VEC>(X + row * a.ldx + col(i), a.D - col(i));
        if (R)
#pragma unroll
            for (int i = 0; i < NV; ++i) r[i] = load8<T, VEC>(R + row * a.ldr + col(i), a.D - col(i));
        float ss[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (R) x[i] = rounded<T, VEC>(values(x[i]) + values(r[i]));
            const f32x8 s = values(x[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) ss[0] = fmaf(s[e], s[e], ss[0]);
        }
        if (a.S)
#pragma unroll
            for (int i = 0; i < NV; ++i) store8<T, VEC>(static_cast<T *>(a.S) + row * a.D + col(i), x[i], a.D - col(i));
        sum(ss);
        const float rho = inverse_root(ss[0] / (float)a.D + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            f32x8 u = values(x[i]);
            if (a.w) u *= values(w[i]);
            if (a.Y) store8<T, VEC>(static_cast<T *>(a.Y) + row * a.D + col(i), rounded<T, VEC>(u * rho), a.D - col(i));
            if (a.Q) {
                // y * 448 / max|y| = u * 448 / max|u|: the row's factor has no part in the 8 bits
                float top = __uint_as_float(top_of_16(top8(u))), ytop = top * rho, least = kTop / kLeast;
                if (top < 0x1p-60f) {      // (next to nothing in a row that is next to nothing: with a small eps these factors leave fp32)
                    u *= 0x1p64f;
                    top *= 0x1p64f;
                    least *= 0x1p-64f;
                }
                // 448 / top as two numbers: one alone is off by two roundings, and what lies at the middle of two steps of e4m3 would go
                // either way
                const float one = 1.f / top;
                float inv = one * kTop, rest = fmaf(-inv, top, kTop) * one, scale = ytop * (1.f / kTop);
                if (ytop < kLeast) {
                    inv = rho * least;
                    rest = 0.f;
                    scale = kLeast / kTop;
                }
                if (!(ytop >= 0.f)) inv = ytop;      // NaN
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = fmaf(u[e], inv, u[e] * rest);
                if (col(i) < a.D) {
                    store_e4m3(static_cast<uint8_t *>(a.Q) + row * a.ldq + col(i), to_e4m3(u), a.D - col(i));
                    if (lane % 16 == 0) a.scale[(long long)(col(i) / 128) * a.M + row] = scale;
                }
            }
        }
    }
}

// dx = ds + rho g - s rho^3 mean(g s); a lane keeps the sums of its columns of dw over the rows that it meets.  Two workgroups to a
// compute unit: their sums are 512 rows more to write and read (one, 8191 x 4096: 62 us instead of 51; four: 54).
template <typename T, bool VEC, int G, int NV>
__global__ __launch_bounds__(kThreads<G>) void norm_bwd_kernel(NormBwd a)
{
    constexpr int rows = kThreads<G> / G;
    __shared__ float part[2][2][16];
    RowSum<G, 2> sum{part};
    const int lane = threadIdx.x % G;
    const T *S = static_cast<const T *>(a.S), *dY = static_cast<const T *>(a.dY), *dS = static_cast<const T *>(a.dS);
    auto col = [&](int i) { return (i * G + lane) * 8; };
    Raw8<T, VEC> w[NV];
    f32x8 dw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        dw[i] = 0.f;
        if (a.w) w[i] = load8<T, VEC>(static_cast<const T *>(a.w) + col(i), a.D - col(i));
    }
    for (long long row = (long long)blockIdx.x * rows + threadIdx.x / G; row < a.M; row += (long long)gridDim.x * rows) {
        Raw8<T, VEC> s[NV], dy[NV], ds[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            s[i] = load8<T, VEC>(S + row * a.lds + col(i), a.D - col(i));
            dy[i] = load8<T, VEC>(dY + row * a.lddy + col(i), a.D - col(i));
            if (dS) ds[i] = load8<T, VEC>(dS + row * a.ldds + col(i), a.D - col(i));
        }
        float t[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const f32x8 sv = values(s[i]);
            f32x8 g = values(dy[i]);
            if (a.w) g *= values(w[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                t[0] = fmaf(sv[e], sv[e], t[0]);
                t[1] = fmaf(g[e], sv[e], t[1]);
            }
        }
        sum(t);
        const float rho = inverse_root(t[0] / (float)a.D + a.eps), back = rho * rho * (t[1] / (float)a.D);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const f32x8 sv = values(s[i]), d = values(dy[i]);
            f32x8 g = d;
            if (a.w) g *= values(w[i]);
            f32x8 dx = (g - sv * back) * rho;
            if (dS) dx += values(ds[i]);
            dw[i] += d * (sv * rho);
            store8<T, VEC>(static_cast<T *>(a.dX) + row * a.D + col(i), rounded<T, VEC>(dx), a.D - col(i));
        }
    }
    if (!a.dw) return;
    if constexpr (rows > 1) {      // the rows of a workgroup meet first, one after the other
        __shared__ float joined[G * NV * 8];
        for (int k = 0; k < rows; ++k) {
            if ((int)threadIdx.x / G == k)
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float &j = joined[col(i) + e];
                        if (k) dw[i][e] += j;
                        if (k < rows - 1) j = dw[i][e];
                    }
            __syncthreads();
        }
        if ((int)threadIdx.x / G != rows - 1) return;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
        store8<float, false>(a.part + (long long)blockIdx.x * a.D + col(i), rounded<float, false>(dw[i]), a.D - col(i));
}

// dw = sum of the workgroups' sums: a workgroup takes 32 columns, 32 slices of the sums side by side, sixteen loads of a slice on
// their way at once.
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float *part, float *dw, int parts, int D)
{
    __shared__ float s[32][33];
    const int x = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float t = 0.f;
    for (int p0 = k; p0 < parts; p0 += 32 * 16) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = c < D && p0 + 32 * i < parts ? part[(long long)(p0 + 32 * i) * D + c] : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) t += v[i];
    }
    s[k][x] = t;
    __syncthreads();
    if (k || c >= D) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) t += s[i][x];
    dw[c] = t;
}

// G lanes and NV steps for rows of D
template <typename F> void by_width(int D, F f)
{
    using std::integral_constant;
    auto go = [&](auto G, auto NV) { f(G, NV); };
#define PF_SHAPE(g, n) return go(integral_constant<int, g>{}, integral_constant<int, n>{})
    if (D <= 128) PF_SHAPE(16, 1);
    if (D <= 256) PF_SHAPE(16, 2);
    if (D <= 512) PF_SHAPE(64, 1);
    if (D <= 1024) PF_SHAPE(64, 2);
    if (D <= 2048) PF_SHAPE(256, 1);
    if (D <= 4096) PF_SHAPE(256, 2);
    if (D <= 8192) PF_SHAPE(1024, 1);
    PF_SHAPE(1024, 2);
#undef PF_SHAPE
}

template <typename T, typename F> void by_type(bool vec, F f)
{
    if (vec) f((T)0.f, std::true_type{});
    else f((T)0.f, std::false_type{});
}

}  // namespace

hipError_t launch_norm_fwd(const NormFwd &a, bool is_bf16, hipStream_t stream)
{
    auto launch = [&](auto one, auto vec) {
        by_width(a.D, [&](auto G, auto NV) {
            using T = decltype(one);
            constexpr int threads = kThreads<G.value>, rows = threads / G.value;
            const long long want = ((long long)a.M + rows - 1) / rows, most = 32LL * device_cu_count();
            hipLaunchKernelGGL((norm_fwd_kernel<T, vec.value, G.value, NV.value>), dim3((unsigned)(want < most ? want : most)),
                               dim3(threads), 0, stream, a);
        });
    };
    const int size = is_bf16 ? 2 : 4;
    const bool vec = a.D % 8 == 0 && wide(a.X, a.ldx, size) && (!a.R || wide(a.R, a.ldr, size));
    if (is_bf16) by_type<bf16>(vec, launch);
    else by_type<float>(vec, launch);
    return hipGetLastError();
}

int norm_bwd_parts(int M, int D)
{
    long long n = 0;
    by_width(D, [&](auto G, auto) {
        constexpr int rows = kThreads<G.value> / G.value;
        const long long want = ((long long)M + rows - 1) / rows, most = 2LL * device_cu_count();
        n = want < most ? want : most;
    });
    return (int)n;
}

hipError_t launch_norm_bwd(const NormBwd &a, bool is_bf16, hipStream_t stream)
{
    const int parts = a.M ? norm_bwd_parts(a.M, a.D) : 0;
    auto launch = [&](auto one, auto vec) {
        by_width(a.D, [&](auto G, auto NV) {
            hipLaunchKernelGGL((norm_bwd_kernel<decltype(one), vec.value, G.value, NV.value>), dim3(parts),
                               dim3(kThreads<G.value>), 0, stream, a);
        });
    };
    const int size = is_bf16 ? 2 : 4;
    const bool vec = a.D % 8 == 0 && wide(a.S, a.lds, size) && wide(a.dY, a.lddy, size) && (!a.dS || wide(a.dS, a.ldds, size));
    if (parts) {
        if (is_bf16) by_type<bf16>(vec, launch);
        else by_type<float>(vec, launch);
    }
    if (a.dw) hipLaunchKernelGGL(norm_dw_kernel, dim3((a.D + 31) / 32), dim3(1024), 0, stream, a.part, a.dw, parts, a.D);
    return hipGetLastError();
}

}  // namespace pf
