// Gated delta rule, one token: S <- a S + beta (v - a S k) k^T, o = S q, in place.  A state is read and written once (128 KB
// for a head of 128 x 128), which is what bounds it.  Sixteen lanes have a row of the state, four rows to a wavefront side by side, and o
// comes from S k, S q and k.q, so that a row is looked at only once:  e = beta (v - a S k),  o = a S q + e k.q.
// 256 sequences of 32 heads of 128 x 128: 221 us, 4.9 TB/s of reading and writing; one sequence 5 us.
#include "pf_gdelta.h"

namespace pf {
namespace gd {
namespace {

// J: d_k in blocks of 64, of which a lane has four consecutive values each; WIDE: rows begin at 16 bytes and are whole.
template <typename T, int J, bool WIDE>
__global__ __launch_bounds__(256) void step_kernel(GDeltaStep a, int rows, int tiles)
{
    constexpr int AT_ONCE = 4;      // rows of a lane under way together
    const int id = blockIdx.x, tile = id % tiles, bh = id / tiles, b = bh / a.Hv, h = bh - b * a.Hv, hk = h / (a.Hv / a.Hk);
    const int l = threadIdx.x & 15, first = tile * rows + (threadIdx.x >> 4), end = min(a.dv, (tile + 1) * rows);
    T *O = static_cast<T *>(a.O) + (long long)bh * a.dv;
    const int slot = a.slots ? a.slots[b] : b;
    // of several sequences with one slot the first is served
    bool taken = false;
    if (a.slots)
        for (int i = threadIdx.x; i < b; i += 256) taken |= a.slots[i] == slot;
    if (a.slots) taken = __syncthreads_or(taken);
    if (slot < 0 || slot >= a.pool || taken) {
        for (int r = first; r < end; r += 16)
            if (l == 0) O[r] = (T)0.f;
        return;
    }
    const T *K = static_cast<const T *>(a.K) + b * a.kb + hk * a.kh, *Q = static_cast<const T *>(a.Q) + b * a.qb + hk * a.qh;
    const T *V = static_cast<const T *>(a.V) + b * a.vb + h * a.vh;
    f32x4 k[J], q[J];
    float kq = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = 64 * j + 4 * l + e;
            const bool in = c < a.dk;
            k[j][e] = in ? to_f32(K[c]) : 0.f;
            q[j][e] = in ? to_f32(Q[c]) : 0.f;
            kq += k[j][e] * q[j][e];
        }
    kq = sum_of_16(kq);
    const float decay = power((double)gate_in(to_f32(static_cast<const T *>(a.G)[b * a.gb + h * a.gh])) * kLog2e);
    const float beta = to_f32(static_cast<const T *>(a.beta)[b * a.bb + h * a.bh]);
    float *S = a.S + ((long long)slot * a.Hv + h) * a.dv * a.dk + 4 * l;

    for (int r0 = first; r0 < end; r0 += 16 * AT_ONCE) {
        f32x4 s[AT_ONCE][J];
        float v[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int r = r0 + 16 * i;
            v[i] = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j) s[i][j] = zero4();
            if (r < end) {
                v[i] = to_f32(V[r]);
                const float *p = S + (long long)r * a.dk;
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    if constexpr (WIDE) {
                        if (64 * j + 4 * l < a.dk) s[i][j] = *reinterpret_cast<const f32x4 *>(p + 64 * j);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (64 * j + 4 * l + e < a.dk) s[i][j][e] = p[64 * j + e];
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int r = r0 + 16 * i;
            float sk = 0.f, sq = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sk += s[i][j][e] * k[j][e], sq += s[i][j][e] * q[j][e];
            const float u = beta * (v[i] - decay * sum_of_16(sk)), o = decay * sum_of_16(sq) + u * kq;
            if (r >= end) continue;
            if (l == 0) O[r] = (T)o;
            float *p = S + (long long)r * a.dk;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const f32x4 n = decay * s[i][j] + u * k[j];
                if constexpr (WIDE) {
                    if (64 * j + 4 * l < a.dk) *reinterpret_cast<f32x4 *>(p + 64 * j) = n;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (64 * j + 4 * l + e < a.dk) p[64 * j + e] = n[e];
                }
            }
        }
    }
}

template <typename T, int J> hipError_t step(const GDeltaStep &a, hipStream_t stream)
{
    // sixteen rows at least to a workgroup (one to each 16 lanes), and more where there are 1024 workgroups without: four rows of a lane are under
    // way together only then
    int rows = 16;
    while (rows < 128 && rows < a.dv && (double)a.B * a.Hv * ((a.dv + 2 * rows - 1) / (2 * rows)) >= 1024) rows *= 2;
    const int tiles = (a.dv + rows - 1) / rows;
    const double groups = (double)a.B * a.Hv * tiles;
    if (!launch_holds(groups, 256)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)groups);
    if (a.dk % 4 == 0) step_kernel<T, J, true><<<grid, 256, 0, stream>>>(a, rows, tiles);
    else step_kernel<T, J, false><<<grid, 256, 0, stream>>>(a, rows, tiles);
    return hipGetLastError();
}
template <typename T> hipError_t step(const GDeltaStep &a, hipStream_t stream)
{
    return a.dk <= 64 ? step<T, 1>(a, stream) : a.dk <= 128 ? step<T, 2>(a, stream) : step<T, 4>(a, stream);
}

}  // namespace
}  // namespace gd

hipError_t launch_gdelta_step(const GDeltaStep &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? gd::step<bf16>(a, stream) : gd::step<float>(a, stream);
}

}  // namespace pf
