// A matrix in 8 bits (e4m3) with scales, as it lies and transposed.
//
// m = max(max|x| over the block, 1e-30), scale = m * (1/448), value = e4m3(x * (1/m * 448)), each operation rounded in fp32.
// A workgroup takes a tile of 128 x 128: a thread eight rows by eight columns in registers, so a row of the tile is sixteen
// lanes, a column sixteen groups of them.  Memory sees x once, whatever is written of it.  Bound by HBM: 8192 x 4096 in bf16, transposed,
// 23 us, 4.4 TB/s; 32768 x 4096 4.8, as it lies 5.1.
#include "pf_layer_common.h"
#include "pf_layer_internal.h"

#include <type_traits>

namespace pf {

namespace {

struct Factor { float inv, scale; };
__device__ __forceinline__ Factor factor_of(uint32_t magnitude)
{
    float m = __uint_as_float(magnitude);
    if (m < kLeast) m = kLeast;
    return {1.f / m * kTop, m * (1.f / kTop)};
}

template <typename T, bool VEC, bool SQUARE, bool PLAIN, bool TURNED>
__global__ __launch_bounds__(256) void quant_kernel(Quant a, int col_tiles)
{
    __shared__ uint32_t tops[4][128];
    __shared__ __attribute__((aligned(16))) uint8_t turned[TURNED ? 128 * 144 : 16];      // rows 144 bytes apart
    const int t = threadIdx.x, c8 = t & 15, r8 = t >> 4;
    const long long row0 = (long long)(blockIdx.x / col_tiles) * 128;
    const int col0 = (int)(blockIdx.x % col_tiles) * 128;
    const int c = col0 + 8 * c8;
    const T *X = static_cast<const T *>(a.X);
    Raw8<T, VEC> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const long long row = row0 + 8 * r8 + i;
        x[i] = load8<T, VEC>(X + row * a.ldx + c, row < a.M ? a.K - c : 0);
    }
    Factor square;
    if constexpr (SQUARE) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, top8(values(x[i])));
        m = top_of_16(m);
        if (c8 == 0) tops[0][r8] = m;
        __syncthreads();
        m = tops[0][0];
        for (int i = 1; i < 16; ++i) m = max(m, tops[0][i]);
        square = factor_of(m);
        const int rt = (int)(row0 / 128), ct = col0 / 128;
        if (t == 0) {
            if (PLAIN) a.scale[(long long)ct * ((a.M + 127LL) / 128) + rt] = square.scale;
            if (TURNED) a.scaleT[(long long)rt * col_tiles + ct] = square.scale;
        }
    }
    if constexpr (PLAIN) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const long long row = row0 + 8 * r8 + i;
            const f32x8 v = values(x[i]);
            Factor f;
            if constexpr (SQUARE) f = square;
            else f = factor_of(top_of_16(top8(v)));
            if (row < a.M) {
                if (c < a.K) store_e4m3(static_cast<uint8_t *>(a.Q) + row * a.ldq + c, to_e4m3(v * f.inv), a.K - c);
                if (!SQUARE && c8 == 0) a.scale[(long long)(col0 / 128) * a.M + row] = f.scale;
            }
        }
    }
    if constexpr (TURNED) {
        float inv[8];
        if constexpr (SQUARE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) inv[e] = square.inv;
        } else {
            uint32_t m[8] = {};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x8 v = values(x[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) m[e] = max(m[e], magnitude(v[e]));
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                m[e] = max(m[e], (uint32_t)__shfl_xor((int)m[e], 16));
                m[e] = max(m[e], (uint32_t)__shfl_xor((int)m[e], 32));
                if ((t & 63) < 16) tops[t >> 6][8 * c8 + e] = m[e];
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = 8 * c8 + e;
                const Factor f = factor_of(max(max(tops[0][k], tops[1][k]), max(tops[2][k], tops[3][k])));
                inv[e] = f.inv;
                if (r8 == 0 && col0 + k < a.K) a.scaleT[(row0 / 128) * a.K + col0 + k] = f.scale;
            }
        }
        f32x8 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = values(x[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f32x8 down;      // eight rows of one column
#pragma unroll
            for (int i = 0; i < 8; ++i) down[i] = v[i][e] * inv[e];
            *reinterpret_cast<u32x2 *>(turned + (8 * c8 + e) * 144 + 8 * r8) = to_e4m3(down);
        }
        __syncthreads();
        // eight lanes write the 128 bytes of a column
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = 32 * i + (t >> 3), r = 16 * (t & 7);
            if (col0 + k >= a.K) continue;
            uint8_t *to = static_cast<uint8_t *>(a.QT) + (long long)(col0 + k) * a.ldqt + row0 + r;
            const u32x4 q = *reinterpret_cast<const u32x4 *>(turned + k * 144 + r);
            if (row0 + r + 16 <= a.M) {
                *reinterpret_cast<u32x4 *>(to) = q;
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (row0 + r + e < a.M) to[e] = (uint8_t)(q[e / 4] >> (8 * (e % 4)));
            }
        }
    }
}

}  // namespace

hipError_t launch_quant(const Quant &a, bool is_bf16, hipStream_t stream)
{
    const int col_tiles = a.K / 128 + (a.K % 128 != 0);
    const long long tiles = ((a.M + 127LL) / 128) * col_tiles;
    if (!launch_holds((double)tiles, 256)) return hipErrorInvalidConfiguration;      // (2^37 values)
    auto launch = [&](auto one, auto vec) {
        auto with = [&](auto square, auto plain, auto turned) {
            hipLaunchKernelGGL((quant_kernel<decltype(one), vec.value, square.value, plain.value, turned.value>),
                               dim3((unsigned)tiles), dim3(256), 0, stream, a, col_tiles);
        };
        auto what = [&](auto square) {
            if (a.Q && a.QT) with(square, std::true_type{}, std::true_type{});
            else if (a.Q) with(square, std::true_type{}, std::false_type{});
            else with(square, std::false_type{}, std::true_type{});
        };
        if (a.rows == 128) what(std::true_type{});
        else what(std::false_type{});
    };
    const bool vec = a.K % 8 == 0 && wide(a.X, a.ldx, is_bf16 ? 2 : 4);
    if (is_bf16) {
        if (vec) launch((bf16)0.f, std::true_type{});
        else launch((bf16)0.f, std::false_type{});
    } else {
        if (vec) launch(0.f, std::true_type{});
        else launch(0.f, std::false_type{});
    }
    return hipGetLastError();
}

}  // namespace pf
