// Norm of every head of queries and keys with the rotation by the token's position, and its backward (include/pf_layer.h).  Memory
// is what bounds both: a row is read once and written once (the backward reads two).  65536 tokens of 64 heads of 128 in bf16, 1.07 GB each
// way: 405 us, 5.3 TB/s (a copy of that size 423); the backward of 16383 tokens of 48 such heads 122 us, 5.0 TB/s.  (With units of eight values,
// so of 8-byte accesses, and four rows of a lane under way: 575 and 193.)
//
// A row of d values is cut into units of sixteen for a lane, two pieces of eight: of the turned ones eight pairs, a and b of a pair in the same
// lane (in halves the pieces lie rot / 2 apart, else side by side), the others as they follow.  So every access is 16 bytes of
// bf16, and of a rotation no value crosses lanes.  64 / LPR rows lie side by side in a wavefront.
#include "pf_layer_common.h"
#include "pf_layer_internal.h"

namespace pf {
namespace {

// over LPR neighbouring lanes
template <int LPR> __device__ __forceinline__ float row_sum(float s)
{
    auto dpp = [](float v, auto ctrl) {
        return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    s += dpp(s, std::integral_constant<int, 0xb1>{});                                // quad_perm 1 0 3 2
    s += dpp(s, std::integral_constant<int, 0x4e>{});                                // quad_perm 2 3 0 1
    if constexpr (LPR >= 8) s += dpp(s, std::integral_constant<int, 0x141>{});       // row_half_mirror
    if constexpr (LPR >= 16) s += dpp(s, std::integral_constant<int, 0x140>{});      // row_mirror
    if constexpr (LPR >= 32) s += __shfl_xor(s, 16);
    if constexpr (LPR >= 64) s += __shfl_xor(s, 32);
    return s;
}

struct Unit {
    int p0, p1, n0, n1, pair;      // two pieces of up to eight values; the first pair's number, or -1
};
__device__ __forceinline__ Unit unit_at(const Heads &a, int u)
{
    const int half = a.rot / 2, turning = (half + 7) / 8;
    Unit x;
    if (u < turning) {
        const int n = min(8, half - 8 * u);      // pairs
        x.pair = 8 * u;
        x.p0 = a.pairs ? 16 * u : 8 * u;
        x.p1 = a.pairs ? 16 * u + 8 : half + 8 * u;
        x.n0 = a.pairs ? min(8, 2 * n) : n;
        x.n1 = a.pairs ? 2 * n - x.n0 : n;
    } else {
        x.pair = -1;
        x.p0 = a.rot + 16 * (u - turning), x.p1 = x.p0 + 8;
        x.n0 = min(8, max(0, a.d - x.p0)), x.n1 = min(8, max(0, a.d - x.p1));
    }
    return x;
}
// Sixteen values as they lie in memory.  VEC: none or eight to a piece, at multiples of 16 bytes.
template <typename T, bool VEC> struct Raw {
    Raw8<T, VEC> a, b;
};
template <typename T, bool VEC> __device__ __forceinline__ Raw<T, VEC> get(const T *p, const Unit &x, bool there)
{
    return {load8<T, VEC>(p + x.p0, there ? x.n0 : 0), load8<T, VEC>(p + x.p1, there ? x.n1 : 0)};
}
template <typename T, bool VEC> __device__ __forceinline__ void set(T *p, const Unit &x, f32x8 a, f32x8 b)
{
    store8<T, VEC>(p + x.p0, rounded<T, VEC>(a), x.n0);
    store8<T, VEC>(p + x.p1, rounded<T, VEC>(b), x.n1);
}
// first and second values of eight pairs out of the two pieces, and back
__device__ __forceinline__ void apart(bool pairs, f32x8 &x, f32x8 &y)
{
    if (!pairs) return;
    const f32x8 a = __builtin_shufflevector(x, y, 0, 2, 4, 6, 8, 10, 12, 14);
    y = __builtin_shufflevector(x, y, 1, 3, 5, 7, 9, 11, 13, 15);
    x = a;
}
__device__ __forceinline__ void together(bool pairs, f32x8 &x, f32x8 &y)
{
    if (!pairs) return;
    const f32x8 a = __builtin_shufflevector(x, y, 0, 8, 1, 9, 2, 10, 3, 11);
    y = __builtin_shufflevector(x, y, 4, 12, 5, 13, 6, 14, 7, 15);
    x = a;
}
// cosines and sines of a unit's pairs at a token's position (NaN where the table has no such position)
template <bool VEC> __device__ __forceinline__ void turns(const Heads &a, const Unit &x, int token, f32x8 &c, f32x8 &s)
{
    c = s = 0.f;
    if (x.pair < 0) return;
    const int at = a.positions[token];
    if (at < 0 || at >= a.far) {
        c = s = __builtin_nanf("");
        return;
    }
    const float *row = a.table + (long long)at * a.rot + x.pair;
    const int n = min(8, a.rot / 2 - x.pair);
    if (VEC && n == 8) c = values(load8<float, VEC>(row, 8)), s = values(load8<float, VEC>(row + a.rot / 2, 8));
    else c = values(load8<float, false>(row, n)), s = values(load8<float, false>(row + a.rot / 2, n));
}
template <typename T, bool VEC> __device__ __forceinline__ void weights(const Heads &a, const HeadSide &side, const Unit &x, f32x8 &u, f32x8 &v)
{
    u = v = 1.f;
    if (!side.w) return;
    const Raw<T, VEC> w = get<T, VEC>(static_cast<const T *>(side.w), x, true);
    u = values(w.a), v = values(w.b);
    apart(a.pairs, u, v);
}
__device__ __forceinline__ float squares(f32x8 u, f32x8 v)
{
    u = u * u + v * v;
    return ((u[0] + u[1]) + (u[2] + u[3])) + ((u[4] + u[5]) + (u[6] + u[7]));
}

// A wavefront has `each` heads of one token, queries and keys one behind the other, and reads the token's cosines and sines once.
template <typename T, int LPR, bool VEC>
__global__ __launch_bounds__(256) void heads_fwd_kernel(Heads a, int groups, int each)
{
    constexpr int ROWS = 64 / LPR, AHEAD = 2;      // AHEAD: rows of a lane under way together
    const int wave = __builtin_amdgcn_readfirstlane((int)((blockIdx.x * 256ll + threadIdx.x) >> 6)), lane = threadIdx.x & 63;
    const int token = wave / groups, first = (wave - token * groups) * each, mine = lane / LPR;
    if (token >= a.M) return;
    const Unit x = unit_at(a, lane % LPR);
    f32x8 c, s;
    turns<VEC>(a, x, token, c, s);
    const float share = a.l2 ? 1.f : 1.f / (float)a.d;
    int before = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const HeadSide &side = a.side[k];
        const int lo = max(first - before, 0), hi = min(first + each - before, side.H);
        before += side.H;
        if (lo >= hi) continue;
        f32x8 wu, wv;
        weights<T, VEC>(a, side, x, wu, wv);
        wu *= side.scale, wv *= side.scale;
        const T *from = static_cast<const T *>(side.X) + token * side.xt + mine * side.xh;
        T *to = static_cast<T *>(side.Y) + ((long long)token * side.H + mine) * a.d;
        for (int h = lo; h < hi; h += ROWS * AHEAD) {
            Raw<T, VEC> r[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) r[i] = get<T, VEC>(from + (h + i * ROWS) * side.xh, x, h + i * ROWS + mine < hi);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                f32x8 u = values(r[i].a), v = values(r[i].b);
                const float rho = 1.f / sqrtf(row_sum<LPR>(squares(u, v)) * share + a.eps);
                if (h + i * ROWS + mine >= hi) continue;
                apart(a.pairs, u, v);
                u *= rho * wu, v *= rho * wv;
                f32x8 y = u, z = v;
                if (x.pair >= 0) y = u * c - v * s, z = u * s + v * c;      // (not 1 and 0 elsewhere: an infinity stays where it is)
                together(a.pairs, y, z);
                set<T, VEC>(to + (long long)(h + i * ROWS) * a.d, x, y, z);
            }
        }
    }
}

// With n the norm's divisor, xh = x / n and g = w times the gradient turned back: dx = (g - xh (mean or sum of g xh)) / n, dw the sum of
// the gradient turned back times xh.  A workgroup has rows of one side; these sums stay with a lane over all of its rows, then one part for
// each workgroup, the queries' first.
template <typename T, int LPR, bool VEC, bool WEIGHTS>
__global__ __launch_bounds__(256) void heads_bwd_kernel(Heads a, int parts0, int each)
{
    constexpr int ROWS = 64 / LPR;
    const int k = (int)blockIdx.x >= parts0, lane = threadIdx.x & 63, mine = lane / LPR;
    const int block = (int)blockIdx.x - (k ? parts0 : 0), blocks = k ? (int)gridDim.x - parts0 : parts0;
    const HeadSide &side = a.side[k];
    const int groups = (side.H + each - 1) / each;
    const Unit x = unit_at(a, lane % LPR);
    f32x8 wu, wv, du = 0.f, dv = 0.f;
    weights<T, VEC>(a, side, x, wu, wv);
    const float share = a.l2 ? 1.f : 1.f / (float)a.d, scale = side.scale;
    const long long items = (long long)a.M * groups;
    for (long long item = (long long)block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); item < items; item += blocks * 4) {
        const int token = (int)(item / groups), lo = (int)(item - (long long)token * groups) * each, hi = min(side.H, lo + each);
        f32x8 c, s;
        turns<VEC>(a, x, token, c, s);
        const T *from = static_cast<const T *>(side.X) + token * side.xt + mine * side.xh;
        const T *grad = static_cast<const T *>(side.dY) + token * side.dyt + mine * side.dyh;
        T *to = static_cast<T *>(side.Y) + ((long long)token * side.H + mine) * a.d;
        for (int h = lo; h < hi; h += ROWS) {
            const bool there = h + mine < hi;
            const Raw<T, VEC> r = get<T, VEC>(from + h * side.xh, x, there), t = get<T, VEC>(grad + h * side.dyh, x, there);
            f32x8 u = values(r.a), v = values(r.b), p = values(t.a), q = values(t.b);
            const float rho = 1.f / sqrtf(row_sum<LPR>(squares(u, v)) * share + a.eps);
            apart(a.pairs, u, v);
            apart(a.pairs, p, q);
            u *= rho, v *= rho;
            p *= scale, q *= scale;
            f32x8 back = p, next = q;
            if (x.pair >= 0) back = p * c + q * s, next = q * c - p * s;
            if constexpr (WEIGHTS)
                if (there) du += back * u, dv += next * v;
            const f32x8 g = back * wu, f = next * wv;
            f32x8 m = g * u + f * v;
            const float along = row_sum<LPR>(((m[0] + m[1]) + (m[2] + m[3])) + ((m[4] + m[5]) + (m[6] + m[7]))) * share;
            if (!there) continue;
            f32x8 y = rho * (g - u * along), z = rho * (f - v * along);
            together(a.pairs, y, z);
            set<T, VEC>(to + (long long)h * a.d, x, y, z);
        }
    }
    if constexpr (WEIGHTS) {
        __shared__ f32x8 sums[4][64][2];
        const int wave = threadIdx.x >> 6;
        sums[wave][lane][0] = du, sums[wave][lane][1] = dv;
        __syncthreads();
        if (threadIdx.x < 2 * LPR) {      // (a piece of a unit: of all rows and wavefronts in their order)
            const int u = threadIdx.x >> 1, piece = threadIdx.x & 1;
            f32x8 all = 0.f;
            for (int r = 0; r < 4 * ROWS; ++r) all += sums[r / ROWS][r % ROWS * LPR + u][piece];
            sums[0][u][piece] = all;      // (its own: row 0 of wavefront 0 has been read)
        }
        __syncthreads();
        if (threadIdx.x < LPR) {
            f32x8 u = sums[0][lane][0], v = sums[0][lane][1];
            together(a.pairs, u, v);
            set<float, false>(a.part + (long long)blockIdx.x * a.d, x, u, v);
        }
    }
}

// dw out of the workgroups' parts: 16 columns to a workgroup, 64 rows of them side by side
__global__ __launch_bounds__(1024) void heads_sum_kernel(Heads a, int parts0, int parts)
{
    __shared__ float sums[64][17];
    const int k = blockIdx.y, n = k ? parts - parts0 : parts0, col = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4;
    float *dw = a.side[k].dw;
    if (!dw) return;
    const float *p = a.part + (long long)(k ? parts0 : 0) * a.d + min(col, a.d - 1);
    float sum = 0.f;
    int i = r;
    for (; i + 3 * 64 < n; i += 4 * 64) {      // (four loads under way together)
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = p[(long long)(i + 64 * j) * a.d];
        sum += (v[0] + v[1]) + (v[2] + v[3]);
    }
    for (; i < n; i += 64) sum += p[(long long)i * a.d];
    sums[r][threadIdx.x & 15] = sum;
    __syncthreads();
    if (threadIdx.x < 16 && col < a.d) {
        float all = 0.f;
#pragma unroll
        for (int j = 0; j < 64; ++j) all += sums[j][threadIdx.x];
        dw[col] = all;
    }
}

// heads that a wavefront takes one after another, so that there are enough wavefronts (8192 fill the chip)
int each_of(int M, int H, int rows)
{
    int each = rows;
    while (each < H && (double)M * ((H + 2 * each - 1) / (2 * each)) >= 8192) each *= 2;
    return each;
}
int lanes_of(int units) { return units <= 4 ? 4 : units <= 8 ? 8 : units <= 16 ? 16 : units <= 32 ? 32 : 64; }

// whole pieces at multiples of 16 bytes (a last unit of four pairs that are neighbours is one; 4099 tokens of 17 heads of 72, 40 turned, fp32: 16.9 us
// without these accesses, 15.9 with)
bool vec(const Heads &a, int size, bool backward)
{
    uintptr_t all = 0;
    long long strides = 0;
    for (const HeadSide &s : a.side) {
        if (!s.H) continue;
        all |= reinterpret_cast<uintptr_t>(s.X), strides |= s.xt | s.xh;
        if (backward) all |= reinterpret_cast<uintptr_t>(s.dY), strides |= s.dyt | s.dyh;
    }
    return a.d % 8 == 0 && a.rot % (a.pairs ? 8 : 16) == 0 && (all | (uintptr_t)(strides * size)) % 16 == 0;
}

struct Parts {
    int queries, all, each;
};
// Workgroups of the backward: as many as there is work for, up to 1024 (four wavefronts to a SIMD), shared out by the heads.
Parts parts_of(int M, int Hq, int Hk, int d, int rot)
{
    if (M <= 0 || Hq + Hk <= 0) return {0, 0, 1};
    const int rows = 64 / lanes_of(head_units(d, rot)), each = each_of(M, Hq + Hk, rows);
    auto of = [&](int H) {
        const double work = ((double)M * ((H + each - 1) / each) + 3) / 4, most = 1024. * H / (Hq + Hk);
        return H == 0 ? 0 : (int)(work < most ? work : most < 1 ? 1 : most);
    };
    return {of(Hq), of(Hq) + of(Hk), each};
}

template <typename T, int LPR> hipError_t forward(const Heads &a, hipStream_t stream)
{
    const int H = a.side[0].H + a.side[1].H, each = each_of(a.M, H, 64 / LPR), groups = (H + each - 1) / each;
    const double blocks = ((double)a.M * groups + 3) / 4;
    if (!launch_holds(blocks, 256)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    if (vec(a, sizeof(T), false)) heads_fwd_kernel<T, LPR, true><<<grid, 256, 0, stream>>>(a, groups, each);
    else heads_fwd_kernel<T, LPR, false><<<grid, 256, 0, stream>>>(a, groups, each);
    return hipGetLastError();
}
template <typename T, int LPR> hipError_t backward(const Heads &a, hipStream_t stream)
{
    const Parts n = parts_of(a.M, a.side[0].H, a.side[1].H, a.d, a.rot);
    const bool v = vec(a, sizeof(T), true), dw = a.side[0].dw || a.side[1].dw;
    if (n.all == 0)      // (no rows: dw are zeros)
        ;
    else if (v)
        dw ? heads_bwd_kernel<T, LPR, true, true><<<n.all, 256, 0, stream>>>(a, n.queries, n.each)
           : heads_bwd_kernel<T, LPR, true, false><<<n.all, 256, 0, stream>>>(a, n.queries, n.each);
    else
        dw ? heads_bwd_kernel<T, LPR, false, true><<<n.all, 256, 0, stream>>>(a, n.queries, n.each)
           : heads_bwd_kernel<T, LPR, false, false><<<n.all, 256, 0, stream>>>(a, n.queries, n.each);
    if (hipError_t e = hipGetLastError()) return e;
    if (dw) heads_sum_kernel<<<dim3((a.d + 15) / 16, 2), 1024, 0, stream>>>(a, n.queries, n.all);
    return hipGetLastError();
}
template <typename T> hipError_t heads(const Heads &a, bool back, hipStream_t stream)
{
    switch (lanes_of(head_units(a.d, a.rot))) {
    case 4: return back ? backward<T, 4>(a, stream) : forward<T, 4>(a, stream);
    case 8: return back ? backward<T, 8>(a, stream) : forward<T, 8>(a, stream);
    case 16: return back ? backward<T, 16>(a, stream) : forward<T, 16>(a, stream);
    case 32: return back ? backward<T, 32>(a, stream) : forward<T, 32>(a, stream);
    default: return back ? backward<T, 64>(a, stream) : forward<T, 64>(a, stream);
    }
}

}  // namespace

int heads_bwd_parts(int M, int Hq, int Hk, int d, int rot) { return parts_of(M, Hq, Hk, d, rot).all; }
hipError_t launch_heads_fwd(const Heads &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? heads<bf16>(a, false, stream) : heads<float>(a, false, stream);
}
hipError_t launch_heads_bwd(const Heads &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? heads<bf16>(a, true, stream) : heads<float>(a, true, stream);
}

}  // namespace pf
