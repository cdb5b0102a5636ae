// Product of two matrices in 8 bits (e4m3), C = A B^T, with a scale for every row and block of 128 of A, and for every row
// (b_rows = 1) or 128 rows of B.
//
// C in bf16: v_mfma_f32_16x16x128_f8f6f4, one instruction for a whole block, so the scales come in between instructions,
// one fp32 fma for each of its results.  It adds eight products at a time aligned to the largest of them and drops what lies 2^-13
// below that (measured: 1.4e-5 of the result's norm for normally distributed values), 1/100 of what the rounding to bf16 costs.
// C in fp32: the values are turned to bf16, which holds every e4m3 number, and go through v_mfma_f32_16x16x32_bf16, whose sums are
// fp32 ones (7e-9 of the norm), four of them to a block.
// A lane (r = l & 15, g = l >> 4) holds 32 values of row r of either operand; which 32 does not matter as long as both
// agree: the 16 bytes from 16 g on and from 64 + 16 g on.  B's rows are the first operand and A's the second, so that a lane's four
// results, rows 4 g .. 4 g + 3 of column r, lie side by side in C.
#include "pf_layer_common.h"
#include "pf_layer_internal.h"

#include <type_traits>

namespace pf {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// 32 values of one row, as the products take them
template <bool EXACT> struct Part;
template <> struct Part<false> {
    i32x8 v;
    __device__ __forceinline__ void set(u32x4 lo, u32x4 hi)
    {
        v = __builtin_bit_cast(i32x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
template <> struct Part<true> {
    bf16x8 v[4];
    __device__ __forceinline__ void set(u32x4 lo, u32x4 hi)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t q = i < 2 ? lo[2 * i + j] : hi[2 * i + j - 4];
                w[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, 1.f, false));
                w[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, 1.f, true));
            }
            v[i] = __builtin_bit_cast(bf16x8, w);
        }
    }
};
__device__ __forceinline__ f32x4 product(const Part<false> &b, const Part<false> &a)
{
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, zero, 0, 0, 0, 0, 0, 0);      // (both e4m3, no scales of its own)
}
__device__ __forceinline__ f32x4 product(const Part<true> &b, const Part<true> &a)
{
    f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) c = mfma16(b.v[i], a.v[i], c);
    return c;
}
// bytes at index >= left become zeros
__device__ __forceinline__ u32x4 keep(u32x4 v, int left)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = left - 4 * i;
        v[i] = n >= 4 ? v[i] : n <= 0 ? 0u : v[i] & ((1u << (8 * n)) - 1);
    }
    return v;
}

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16 *p, float v) { *p = (bf16)v; }

// Few rows of A: the weights are what is read, once, straight into registers.  A workgroup takes 16 rows of B and 16 MT of
// A; its eight wavefronts share the blocks of K between them and join their sums at the end, in their order.
template <typename TO, int MT>      // (TO: float is also what asks for exact products)
__global__ __launch_bounds__(512) void matmul_rows_kernel(Matmul a)
{
    __shared__ f32x4 sums[8][MT][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const long long n0 = (long long)blockIdx.x * 16, m0 = (long long)blockIdx.y * (16 * MT);
    const int nk = a.K / 128 + (a.K % 128 != 0), last = (a.K + 15) / 16 * 16 - 16;
    const long long sb_ld = a.b_rows == 1 ? a.N : (a.N + 127LL) / 128;
    const uint8_t *B = static_cast<const uint8_t *>(a.B) + min(n0 + r, (long long)a.N - 1) * a.ldb;
    const uint8_t *A[MT];
    long long m[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        m[i] = min(m0 + 16 * i + r, (long long)a.M - 1);
        A[i] = static_cast<const uint8_t *>(a.A) + m[i] * a.lda;
    }
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = 0.f;
    auto load = [&](const uint8_t *p, int kb, bool cut) {
        const int k0 = kb * 128 + 16 * g, k1 = k0 + 64;
        u32x4 lo = *reinterpret_cast<const u32x4 *>(p + min(k0, last)), hi = *reinterpret_cast<const u32x4 *>(p + min(k1, last));
        if (cut) lo = keep(lo, a.K - k0), hi = keep(hi, a.K - k1);
        Part<sizeof(TO) == 4> part;
        part.set(lo, hi);
        return part;
    };
    auto step = [&](int kb, bool cut) {
        const auto b = load(B, kb, cut);
        f32x4 sb;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const long long n = min(n0 + 4 * g + e, (long long)a.N - 1);
            sb[e] = a.sb[kb * sb_ld + (a.b_rows == 1 ? n : n / 128)];
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const f32x4 p = product(b, load(A[i], kb, cut));
            acc[i] += p * (sb * a.sa[(long long)kb * a.M + m[i]]);
        }
    };
    for (int kb = w; kb < nk; kb += 8) step(kb, kb * 128 + 128 > a.K);
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[w][i][lane] = acc[i];
    __syncthreads();
    TO *C = static_cast<TO *>(a.C);
    for (int i = w; i < MT; i += 8) {
        f32x4 t = sums[0][i][lane];
#pragma unroll
        for (int k = 1; k < 8; ++k) t += sums[k][i][lane];
        const long long row = m0 + 16 * i + r, col = n0 + 4 * g;
        if (row < a.M)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < a.N) put(C + row * a.ldc + col + e, t[e]);
    }
}

}  // namespace

size_t matmul_workspace_bytes(int, int, int, int) { return 0; }

hipError_t launch_matmul(const Matmul &a, bool bf16_out, hipStream_t stream)
{
    auto launch = [&](auto one) {
        auto rows = [&](auto MT) {
            hipLaunchKernelGGL((matmul_rows_kernel<decltype(one), MT.value>),
                               dim3((a.N + 15) / 16, (unsigned)((a.M + 16LL * MT.value - 1) / (16 * MT.value))), dim3(512), 0, stream, a);
        };
        if (a.M <= 16) rows(std::integral_constant<int, 1>{});
        else rows(std::integral_constant<int, 4>{});
    };
    if (bf16_out) launch((bf16)0.f);
    else launch(0.f);
    return hipGetLastError();
}

}  // namespace pf
