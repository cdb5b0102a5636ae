// Gated linear recurrence h_t = a_t h_{t-1} + b_t for every sequence and channel, and its backward.
#include "pf_layer_common.h"
#include "pf_layer_internal.h"

#include <type_traits>

namespace pf {

namespace {

// the decay a, 1 - a, and d a / d g of a gate's value
struct Gate { float a, rest, slope; };
__device__ __forceinline__ Gate gate_of(float g, int form)
{
    if (form == 0) return {g, 1.f - g, 1.f};
    if (form == 1) {
        const float a = expf(g);
        return {a, -expm1f(g), a};
    }
    const float a = 1.f / (1.f + expf(-g)), rest = 1.f / (1.f + expf(g));
    return {a, rest, a * rest};
}

template <typename T>
__global__ __launch_bounds__(64) void gated_fwd_kernel(Gated a)
{
    const int groups = (a.D + 63) / 64, b = blockIdx.x / groups, c = (blockIdx.x % groups) * 64 + threadIdx.x;
    if (c >= a.D) return;
    const T *X = static_cast<const T *>(a.X) + b * a.xb + c, *G = static_cast<const T *>(a.G) + b * a.gb + c;
    T *Y = static_cast<T *>(a.Y) + (long long)b * a.L * a.D + c;
    const long long s = (long long)b * a.D + c;
    float h = a.h0 ? a.h0[s] : 0.f;
#pragma unroll 8
    for (long long t = 0; t < a.L; ++t) {
        const Gate k = gate_of((float)G[t * a.gt], a.gate);
        const float x = (float)X[t * a.xt];
        h = fmaf(k.a, h, a.mix ? k.rest * x : x);
        Y[t * a.D] = (T)h;
    }
    if (a.hL) a.hL[s] = h;
}

template <typename T>
__global__ __launch_bounds__(64) void gated_bwd_kernel(Gated a)
{
    const int groups = (a.D + 63) / 64, b = blockIdx.x / groups, c = (blockIdx.x % groups) * 64 + threadIdx.x;
    if (c >= a.D) return;
    const T *X = static_cast<const T *>(a.X) + b * a.xb + c, *G = static_cast<const T *>(a.G) + b * a.gb + c;
    const T *dY = static_cast<const T *>(a.dY) + b * a.dyb + c;
    const long long at = (long long)b * a.L * a.D + c, s = (long long)b * a.D + c;
    const T *Y = static_cast<const T *>(a.Yin) + at;
    T *dX = static_cast<T *>(a.dX) + at, *dG = static_cast<T *>(a.dG) + at;
    const float h0 = a.h0 ? a.h0[s] : 0.f;
    float back = a.dhL ? a.dhL[s] : 0.f;      // a_{t+1} l_{t+1}
#pragma unroll 8
    for (long long t = a.L - 1; t >= 0; --t) {
        const Gate k = gate_of((float)G[t * a.gt], a.gate);
        const float l = (float)dY[t * a.dyt] + back;
        float h = t > 0 ? (float)Y[(t - 1) * a.D] : h0;
        if (a.mix) h -= (float)X[t * a.xt];
        dX[t * a.D] = (T)(a.mix ? k.rest * l : l);
        dG[t * a.D] = (T)(l * h * k.slope);
        back = k.a * l;
    }
    if (a.dh0) a.dh0[s] = back;
}

}  // namespace

size_t gated_workspace_bytes(int, int, int, bool) { return 0; }

hipError_t launch_gated_fwd(const Gated &a, bool is_bf16, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.B * (long long)((a.D + 63) / 64)));
    if (is_bf16) hipLaunchKernelGGL(gated_fwd_kernel<bf16>, grid, dim3(64), 0, stream, a);
    else hipLaunchKernelGGL(gated_fwd_kernel<float>, grid, dim3(64), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_gated_bwd(const Gated &a, bool is_bf16, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.B * (long long)((a.D + 63) / 64)));
    if (is_bf16) hipLaunchKernelGGL(gated_bwd_kernel<bf16>, grid, dim3(64), 0, stream, a);
    else hipLaunchKernelGGL(gated_bwd_kernel<float>, grid, dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace pf
