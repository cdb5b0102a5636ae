// Gated delta rule: plan of packed sequences, and the flow of every chunk by itself (pf_gdelta.h): T, P and the decays.
#include "pf_gdelta.h"

namespace pf {
namespace gd {
namespace {

// Starts and lengths of packed sequences from their offsets, which are brought into order and into the array first (each is
// at least the largest before it, and no more than there are rows), so that no two sequences share a chunk or a row and there are
// never more chunks than the workspace was sized for.  One workgroup; the sums run over 1024 sequences at a time.
__global__ __launch_bounds__(1024) void plan_kernel(GDelta a)
{
    __shared__ int smem[2][1024];
    __shared__ int carry[2];      // largest offset so far, chunks so far
    const Plan p = plan_of(a.plan, a.N);
    const int t = threadIdx.x;
    if (t == 0) carry[0] = carry[1] = 0;
    __syncthreads();
    for (int base = 0; base < a.N; base += 1024) {
        const int n = base + t, span = min(1024, a.N - base);
        auto offset = [&](int i) { return i <= a.N ? min(max(a.offsets[i], 0), a.L) : 0; };
        // the largest offset up to n: a running maximum, side by side
        int best = n < a.N ? offset(n) : 0;
        smem[0][t] = best;
        __syncthreads();
        for (int s = 1; s < span; s *= 2) {
            const int other = t >= s ? smem[0][t - s] : 0;
            __syncthreads();
            best = max(best, other);
            smem[0][t] = best;
            __syncthreads();
        }
        const int start = max(best, carry[0]);
        const int last = n < a.N ? max(start, offset(n + 1)) : start;
        const int len = last - start, mine = (len + C - 1) / C;
        int sum = mine;
        smem[1][t] = sum;
        __syncthreads();
        for (int s = 1; s < span; s *= 2) {
            const int other = t >= s ? smem[1][t - s] : 0;
            __syncthreads();
            sum += other;
            smem[1][t] = sum;
            __syncthreads();
        }
        if (n < a.N) p.start[n] = start, p.len[n] = len, p.first[n] = carry[1] + sum - mine;
        __syncthreads();
        if (t == span - 1) carry[0] = max(carry[0], best), carry[1] += sum;
        __syncthreads();
    }
    const int there = carry[1];
    __threadfence_block();
    __syncthreads();
    for (int id = t; id < a.chunks; id += 1024) {
        int lo = 0, hi = a.N - 1;      // the last sequence whose first chunk is not behind id
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (p.first[mid] <= id) lo = mid;
            else hi = mid - 1;
        }
        p.of[id] = id < there ? lo : -1;
    }
}

// A matrix in LDS (TURNED: its transpose) as fragments in NP bf16 parts.
template <int NP, bool TURNED> __device__ __forceinline__ void put_matrix(const float *tile, int ld, bf16 *to)
{
#pragma unroll
    for (int u0 = 0; u0 < 384; u0 += 256) {
        const int u = u0 + threadIdx.x, f = u >> 6, lane = u & 63;
        if (u >= 384) break;
        const int w = TURNED ? (f < 4 ? f >> 1 : f - 2) : f < 2 ? f : (f + 2) >> 1, t = TURNED ? (f < 4 ? f & 1 : 1) : f < 2 ? 0 : f & 1;
        const int row = 16 * w + (lane & 15), col = 32 * t + 8 * (lane >> 4);
        f32x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = TURNED ? tile[(col + e) * ld + row] : tile[row * ld + col + e];
        bf16x8 p[NP];
        split<NP, 8>(v, p);
#pragma unroll
        for (int i = 0; i < NP; ++i) st8(to + ((f * 3 + i) * 64 + lane) * 8, p[i]);
    }
}

// One workgroup of four wavefronts for each chunk and value head; wavefront w has the rows 16 w ..  What it cannot do without is
// reading K and Q (32 KB at d_k = 128 in bf16) and writing T and P (36 KB of fragments): 32768 of them in 400 us, 5.6 TB/s of which heads that
// share rows in a cache line spare some.  The inverse is taken by blocks of 16, on the diagonal a column to a lane, so that only
// 16 steps and three products come one from the other.
template <typename T, int DK, bool FULL, bool BACKWARD>
__global__ __launch_bounds__(256) void flow_kernel(GDelta a)
{
    constexpr int KP = pitch<T>(DK), AP = C + 4, KS = DK / 32, kTokens = C * KP * (int)sizeof(T), kTile = C * AP * 4;
    __shared__ __attribute__((aligned(16))) char smem[kTokens > kTile ? kTokens : kTile];
    __shared__ __attribute__((aligned(16))) float A[C * AP];
    __shared__ __attribute__((aligned(16))) float diag[C * 20];
    __shared__ float coarse[C], fine[C], sbeta[C];
    T *Ks = reinterpret_cast<T *>(smem);
    float *P = reinterpret_cast<float *>(smem);      // in K's place

    const int id = (int)xcd_consecutive(blockIdx.x, gridDim.x), chunk = id / a.Hv, h = id - chunk * a.Hv, hk = h / (a.Hv / a.Hk);
    Chunk x;
    if (!chunk_at(a, chunk, x)) return;
    const int w = wave_id(), lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
    const long long xi = (long long)chunk * a.Hv + h;

    // K into LDS; rows behind the sequence's end are its last row again (their beta is 0, so that they change nothing)
    const T *K = static_cast<const T *>(a.K) + x.seq * a.kb + x.tok * a.kt + hk * a.kh;
    constexpr int UNITS = C * DK / 8 / 256;
    In<T> kr[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int u = i * 256 + threadIdx.x, row = u / (DK / 8), k = 8 * (u % (DK / 8));
        kr[i] = fetch<T, FULL>(K + min(row, x.len - 1) * a.kt + k, a.dk - k);
    }
    In<T> qf[KS];
    const T *Q = static_cast<const T *>(a.Q) + x.seq * a.qb + x.tok * a.qt + hk * a.qh + min(16 * w + r16, x.len - 1) * a.qt;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = fetch<T, FULL>(Q + 32 * s + 8 * g, a.dk - 32 * s - 8 * g);
    if (w == 0) {
        const bool in = lane < x.len;
        const long long t = x.tok + min(lane, x.len - 1);
        const float gate = to_f32(static_cast<const T *>(a.G)[x.seq * a.gb + t * a.gt + h * a.gh]);
        const float beta = in ? to_f32(static_cast<const T *>(a.beta)[x.seq * a.bb + t * a.bt + h * a.bh]) : 0.f;
        double G = in ? (double)gate_in(gate) * kLog2e : 0.;      // sums in fp64: what counts are differences, of far sums too
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const double other = __shfl_up(G, s);
            if (lane >= s) G += other;
        }
        const double whole = __shfl(G, 63);
        const float c = coarse_of(G), f = (float)(G - c);
        coarse[lane] = c, fine[lane] = f, sbeta[lane] = beta;
        float *v = a.vec + xi * kVec;
        v[lane] = power(G);
        v[C + lane] = power(whole - G);
        v[2 * C + lane] = beta;
        v[3 * C + lane] = c;
        v[4 * C + lane] = f;
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int u = i * 256 + threadIdx.x;
        __builtin_memcpy(__builtin_assume_aligned(Ks + u / (DK / 8) * KP + 8 * (u % (DK / 8)), 16), &kr[i], sizeof(kr[i]));
    }
    __syncthreads();

    f32x4 kk[4], qk[4];
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) kk[ct] = qk[ct] = zero4();
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const In<T> ka = frag_rows(Ks, KP, 16 * w + r16, 32 * s + 8 * g);
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
            if (ct > w) continue;
            const In<T> kb = frag_rows(Ks, KP, 16 * ct + r16, 32 * s + 8 * g);
            kk[ct] = mma(ka, kb, kk[ct]);
            qk[ct] = mma(qf[s], kb, qk[ct]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
        const int j = 16 * ct + r16;
        if (ct <= w) {
            const float cj = coarse[j], fj = fine[j];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 16 * w + 4 * g + e;
                const float D = power(coarse[i] - cj, fine[i] - fj);
                A[i * AP + j] = j < i ? sbeta[i] * (D * kk[ct][e]) : 0.f;
                P[i * AP + j] = j <= i ? D * qk[ct][e] : 0.f;
            }
        } else if (ct == w + 1 && (w & 1) == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) P[(16 * w + 4 * g + e) * AP + j] = 0.f;
        }
    }
    __syncthreads();

    // inverse of the diagonal block of 16: lane r16 a column, row after row (all four groups of lanes alike)
    float v[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        float sum = r == r16 ? 1.f : 0.f;
#pragma unroll
        for (int q = 0; q < (r + 3) / 4; ++q) {
            const f32x4 row = *reinterpret_cast<const f32x4 *>(&A[(16 * w + r) * AP + 16 * w + 4 * q]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (4 * q + e < r) sum -= row[e] * v[4 * q + e];
        }
        v[r] = sum;
    }
    f32x4 own;      // as an accumulator tile: rows 4 g ..
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        own[e] = g == 0 ? v[e] : g == 1 ? v[4 + e] : g == 2 ? v[8 + e] : v[12 + e];
        diag[(16 * w + 4 * g + e) * 20 + r16] = own[e];
    }
    __syncthreads();
    // below the diagonal, a column of blocks to a wavefront: T_ij = -T_ii sum over k of A_ik T_kj; a tile that was computed is the next
    // product's right operand as it stands
    f32x4 t[4];
    auto column = [&](auto col) {
        constexpr int J = decltype(col)::value;
        t[J] = own;
#pragma unroll
        for (int i = J + 1; i < 4; ++i) {
            f32x4 X = zero4();
#pragma unroll
            for (int k = J; k < i; ++k) X = mma4(*reinterpret_cast<const f32x4 *>(&A[(16 * i + r16) * AP + 16 * k + 4 * g]), t[k], X);
            t[i] = -mma4(*reinterpret_cast<const f32x4 *>(&diag[(16 * i + r16) * 20 + 4 * g]), X, zero4());
        }
    };
    if (w == 0) column(std::integral_constant<int, 0>{});
    else if (w == 1) column(std::integral_constant<int, 1>{});
    else if (w == 2) column(std::integral_constant<int, 2>{});
    else column(std::integral_constant<int, 3>{});
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i < w && !(i == w - 1 && (w & 1))) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) A[(16 * i + 4 * g + e) * AP + 16 * w + r16] = i < w ? 0.f : t[i][e];
    }
    __syncthreads();
    put_matrix<3, false>(A, AP, a.T + xi * kMatrix);
    if constexpr (BACKWARD) {
        put_matrix<3, true>(A, AP, a.Tt + xi * kMatrix);
        put_matrix<3, true>(P, AP, a.P + xi * kMatrix);
    } else {
        put_matrix<sizeof(T) == 2 ? 2 : 3, false>(P, AP, a.P + xi * kMatrix);
    }
}

template <typename T, int DK> hipError_t flow(const GDelta &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((long long)a.chunks * a.Hv));
    const bool full = gdelta_full(a, sizeof(T));
    if (a.Tt) full ? flow_kernel<T, DK, true, true><<<grid, 256, 0, stream>>>(a) : flow_kernel<T, DK, false, true><<<grid, 256, 0, stream>>>(a);
    else full ? flow_kernel<T, DK, true, false><<<grid, 256, 0, stream>>>(a) : flow_kernel<T, DK, false, false><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t flow(const GDelta &a, hipStream_t stream)
{
    return a.dk <= 64 ? flow<T, 64>(a, stream) : a.dk <= 128 ? flow<T, 128>(a, stream) : flow<T, 256>(a, stream);
}

}  // namespace
}  // namespace gd

size_t gdelta_workspace(GDelta &a, bool backward, void *at)
{
    size_t bytes = 0;
    auto part = [&](auto *&p, size_t count) {
        if (at) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(static_cast<char *>(at) + bytes);
        bytes += (count * sizeof(*p) + 255) / 256 * 256;
    };
    const size_t x = (size_t)a.chunks * a.Hv, dv = (size_t)(a.dv + 31) / 32 * 32;
    if (a.offsets) part(a.plan, 3 * (size_t)a.N + a.chunks);
    part(a.vec, x * gd::kVec);
    part(a.T, x * gd::kMatrix);
    part(a.P, x * gd::kMatrix);
    if (a.segments > 1) {
        const size_t each = (size_t)a.N * a.Hv * a.segments * gdelta_width(a.dk);
        part(a.ends, each * (dv + gdelta_width(a.dk)));
        part(a.starts, each * dv);
        if (backward) part(a.fronts, each * dv);
    }
    if (backward) {
        part(a.Tt, x * gd::kMatrix);
        part(a.S, x * gdelta_state(a));
        part(a.R, x * gdelta_state(a));
        part(a.U, x * gd::C * dv);
        part(a.Z, x * gd::C * dv);
    }
    return bytes;
}

hipError_t launch_gdelta_flow(const GDelta &a, bool is_bf16, hipStream_t stream)
{
    if (a.offsets) {
        gd::plan_kernel<<<1, 1024, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return is_bf16 ? gd::flow<bf16>(a, stream) : gd::flow<float>(a, stream);
}

hipError_t launch_gdelta_fwd(const GDelta &a, bool is_bf16, hipStream_t stream)
{
    if (a.chunks > 0)
        if (hipError_t e = launch_gdelta_flow(a, is_bf16, stream)) return e;
    return launch_gdelta_scan(a, is_bf16, false, stream);
}
hipError_t launch_gdelta_bwd(const GDelta &a, bool is_bf16, hipStream_t stream)
{
    if (a.chunks > 0) {
        if (hipError_t e = launch_gdelta_flow(a, is_bf16, stream)) return e;
        if (hipError_t e = launch_gdelta_scan(a, is_bf16, true, stream)) return e;
    }
    if (hipError_t e = launch_gdelta_scan_bwd(a, is_bf16, stream)) return e;
    return a.chunks > 0 ? launch_gdelta_grad(a, is_bf16, stream) : hipSuccess;
}

}  // namespace pf
