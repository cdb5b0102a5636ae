// Device-side building blocks of the operators around the delta rule: eight values of a row at a time, sums over lanes,
// e4m3 conversion.
#pragma once
#include "pf_common.h"

namespace pf {

typedef float f32x8 __attribute__((ext_vector_type(8)));

// whether rows from p on, `ld` elements of `size` bytes apart, begin at whole 16 bytes
inline bool wide(const void *p, long long ld, int size) { return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) % 16 == 0; }

// Eight consecutive values of a row of which `left` are there (more than 8: all; none: zeros).  VEC: their address is a multiple
// of 16 and `left` is 0 or at least 8; else eight are still one access, which the hardware takes at any address.
template <typename T, bool VEC> struct Raw8;      // as they lie in memory, on their way
template <bool VEC> struct Raw8<bf16, VEC> { u32x4 v; };
template <bool VEC> struct Raw8<float, VEC> { f32x4 v[2]; };

template <typename T, bool VEC> __device__ __forceinline__ Raw8<T, VEC> load8(const T *p, int left)
{
    Raw8<T, VEC> r = {};
    if constexpr (VEC) {
        if (left > 0) __builtin_memcpy(&r, __builtin_assume_aligned(p, 16), sizeof(r));
    } else if (left >= 8) {
        __builtin_memcpy(&r, p, sizeof(r));
    } else if (left > 0) {
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < left ? p[i] : (T)0.f;
        __builtin_memcpy(&r, e, sizeof(r));
    }
    return r;
}
template <bool VEC> __device__ __forceinline__ f32x8 values(const Raw8<bf16, VEC> &r)
{
    f32x8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(r.v[i] << 16);
        f[2 * i + 1] = __uint_as_float(r.v[i] & 0xffff0000u);
    }
    return f;
}
template <bool VEC> __device__ __forceinline__ f32x8 values(const Raw8<float, VEC> &r)
{
    return __builtin_shufflevector(r.v[0], r.v[1], 0, 1, 2, 3, 4, 5, 6, 7);
}
template <typename T, bool VEC> __device__ __forceinline__ Raw8<T, VEC> rounded(f32x8 f)
{
    Raw8<T, VEC> r;
    if constexpr (sizeof(T) == 4) {
        r.v[0] = __builtin_shufflevector(f, f, 0, 1, 2, 3);
        r.v[1] = __builtin_shufflevector(f, f, 4, 5, 6, 7);
    } else {
        typedef bf16 b8 __attribute__((ext_vector_type(8)));
        r.v = __builtin_bit_cast(u32x4, __builtin_convertvector(f, b8));
    }
    return r;
}
template <typename T, bool VEC> __device__ __forceinline__ void store8(T *p, const Raw8<T, VEC> &r, int left)
{
    if constexpr (VEC) {
        if (left > 0) __builtin_memcpy(__builtin_assume_aligned(p, 16), &r, sizeof(r));
    } else if (left >= 8) {
        __builtin_memcpy(p, &r, sizeof(r));
    } else if (left > 0) {
        T e[8];
        __builtin_memcpy(e, &r, sizeof(r));
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = e[i];
    }
}

// fp32 -> e4m3, round to nearest even; beyond 448: NaN
__device__ __forceinline__ u32x2 to_e4m3(f32x8 f)
{
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
        r[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w, true);
    }
    return r;
}
// p: 8-byte aligned (rows of e4m3 lie a multiple of 16 bytes apart)
__device__ __forceinline__ void store_e4m3(uint8_t *p, u32x2 q, int left)
{
    if (left >= 8) {
        *reinterpret_cast<u32x2 *>(p) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
    }
}

constexpr float kTop = 448.f, kLeast = 1e-30f;

// |x| as an unsigned number: ordered as the values are, NaN above infinity, so that the largest of several is NaN if one is
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t top8(f32x8 f)
{
    uint32_t m = magnitude(f[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = max(m, magnitude(f[i]));
    return m;
}
// over the 16 lanes of a DPP row
__device__ __forceinline__ uint32_t top_of_16(uint32_t m)
{
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true));       // quad_perm 1 0 3 2
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, true));       // quad_perm 2 3 0 1
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x124, 0xf, 0xf, true));      // row_ror:4
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x128, 0xf, 0xf, true));   // row_ror:8
}
__device__ __forceinline__ float sum_of_16(float s)
{
    auto dpp = [](float v, auto ctrl) {
        return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    s += dpp(s, std::integral_constant<int, 0xb1>{});
    s += dpp(s, std::integral_constant<int, 0x4e>{});
    s += dpp(s, std::integral_constant<int, 0x124>{});
    return s + dpp(s, std::integral_constant<int, 0x128>{});
}

}  // namespace pf
