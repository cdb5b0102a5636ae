// Gated linear recurrence h_t = a_t h_{t-1} + b_t for every sequence and channel, and its backward, whose recurrence runs
// the other way: with m = a_{t+1} l_{t+1} coming in, l_t = dy_t + m and a_t l_t goes out.
//
// A span of steps takes what comes in, v, to A v + H: A the product of its gates, H what it makes of zero.  Spans join as
// (A, H) then (A', H') = (A' A, A' H + H'), so they can be read side by side.  A is kept as m 2^e: with gates of 2 and then 1/2 it
// leaves fp32 where no state does, and from then on it would be lost.  A wavefront holds 64 V channels of some
// consecutive steps in registers, a workgroup kWaves such spans, one behind the other: a tile.  Each span's (A, H) is formed first, the
// spans in front are put through it, and the steps run once more from what really comes in.  Memory sees every array once.
//
// Three kernels: a few tokens, a lane through all of them; many sequences and channels, a workgroup along a chain (64 V
// channels of one sequence) from tile to tile; else every tile has a workgroup.  A tile tells the (A, H) of its channels as soon as
// it has read them, looks back for the nearest tile in front whose outgoing values are told (each of its wavefronts listens to one
// of the eight in front, where there are few chains to two of sixteen), runs these through the (A, H) of the tiles between, and tells
// its own outgoing values.  A word that is told stands for itself (clear is a pattern that no value has), one store of 4 or 8 bytes, so
// no fence orders anything.  Tiles are handed out by a counter, all chains' first tiles first: a workgroup waits only for tiles handed
// out before its own, whose workgroups are on the chip already and wait for nothing later, so every wait ends.  What a tile makes of
// the values that come in depends on the tiles between them in order, whichever were told, so the bits do not depend on timing.
//
// Bound by HBM: 1 x 65536 x 4096 forward in bf16 325 us, 5.0 TB/s (a plain copy: 5.1); 1 x 65536 x 2048 in fp32 298 us, 5.4 TB/s; backward with
// the mix 2 x 8192 x 4096 192 us, 4.2 TB/s, where the tiles are not long enough for what a tile waits to be hidden.  A long sequence of few
// channels is bound by the chain, 0.19 us a tile: 1 x 65536 x 64 64 us.  Tried and left, where 1 x 65536 x 4096 took 321 us: two channels more to a
// lane (375), workgroups that draw tile after tile and read ahead (475: what they hold in registers makes tiles short), 16 tiles listened to
// here too (twice the words to read: 351), four or twelve wavefronts (363, 348).
#include "pf_layer_common.h"
#include "pf_layer_internal.h"

#include <algorithm>
#include <climits>
#include <type_traits>

namespace pf {

namespace {

constexpr int kWaves = 8, kWalkSteps = 16;
// Steps of a wavefront's span of a tile, as its registers allow: forward (two arrays) two workgroups to a compute unit, of tiles that are
// long, so that there is less to tell and to wait for (1 x 65536 x 4096, bf16: 16 steps 372 us, 24 338, 28 326, 32 329); backward (up to four
// arrays) three of short ones (2 x 8192 x 4096 with the mix: two of 16 steps 197 us, three of 9 193; 16 x 2048 x 4096 386 and 376).
template <typename T, bool BACK, bool MIX, bool FARTHER>
constexpr int kTileSteps = BACK ? (FARTHER ? 16 : 9) : sizeof(T) == 4 ? 32 : FARTHER ? 24 : MIX ? 20 : 28;
template <typename T, bool BACK, bool MIX> constexpr int tile_tokens(bool farther)
{
    return kWaves * (farther ? kTileSteps<T, BACK, MIX, true> : kTileSteps<T, BACK, MIX, false>);
}

// the decay a, 1 - a, and d a / d g of a gate's value
struct Gate { float a, rest, slope; };
// e^x.  x log2 e is rounded, which is |x| / 2 units of fp32 in the result: of gates in fp32 it is put right (1 x 65536 x 2048 296 -> 298 us), gates in bf16
// are themselves off by some 2^15 times that.
template <bool EXACT> __device__ __forceinline__ float exponential(float x)
{
    const float t = x * 1.44269504088896341f, y = __builtin_amdgcn_exp2f(t);
    if constexpr (!EXACT) return y;
    const float rest = fmaf(x, 1.92596298909109e-8f, fmaf(x, 1.44269504088896341f, -t));
    return fabsf(t) < 200.f ? fmaf(y, rest * 0.693147180559945309f, y) : y;      // (infinite x: 0 and infinity)
}
// what is not used of the result is not computed
template <int FORM, bool MIX, bool EXACT> __device__ __forceinline__ Gate gate_of(float g)
{
    if (FORM == 0) return {g, 1.f - g, 1.f};
    if (FORM == 1) {
        const float a = exponential<EXACT>(g);
        float rest = 0.f;
        if (MIX) {      // 1 - e^g: near zero the series, whose first term left out is 2e-8 of it
            float p = 1.f / 5040;
            p = fmaf(p, g, 1.f / 720);
            p = fmaf(p, g, 1.f / 120);
            p = fmaf(p, g, 1.f / 24);
            p = fmaf(p, g, 1.f / 6);
            p = fmaf(p, g, 0.5f);
            p = fmaf(p, g, 1.f);
            rest = fabsf(g) < 0.35f ? -p * g : 1.f - a;
        }
        return {a, rest, a};
    }
    const float e = exponential<EXACT>(-fabsf(g)), d = 1.f + e, near = __builtin_amdgcn_rcpf(d);
    const float s = fmaf(fmaf(-d, near, 1.f), near, near), t = e * s;      // (one step of Newton: 1 / d but for the last rounding)
    return {g < 0.f ? t : s, g < 0.f ? s : t, t * s};
}

// A product of gates, m 2^e: while it is formed 1/2 <= |m| < 1 (or zero, infinite, NaN), when it is used 1 <= |m| < 2, so that 2^e v is
// beyond fp32 only where the whole is.  What that costs, against a product that is one number: 1 x 65536 x 4096 in bf16 317 -> 326 us.
struct Product {
    float m = 0.5f;
    int e = 1;
    __device__ __forceinline__ void times(float a)
    {
        const float n = m * a;
        m = __builtin_amdgcn_frexp_mantf(n);
        e += __builtin_amdgcn_frexp_expf(n);
    }
    __device__ __forceinline__ void ready() { m += m, --e; }
};
// what a span makes of v
__device__ __forceinline__ float through(float m, int e, float H, float v) { return fmaf(m, __builtin_ldexpf(v, e), H); }

// the powers of V neighbouring channels in one word, which is never clear (below)
constexpr int kPowerZero = 1 << 14;
template <int V> __device__ __forceinline__ uint32_t powers(const Product (&A)[V])
{
    const uint32_t w = A[0].e + kPowerZero;      // (32 steps: 4800 at most)
    if constexpr (V == 2) return w | (uint32_t)(A[1].e + kPowerZero) << 16;
    return w;
}
__device__ __forceinline__ int power(uint32_t w, int v) { return (int)(w >> (16 * v) & 0xffff) - kPowerZero; }

// V neighbouring channels of one token
template <typename T, int V> struct Raw { uint32_t w[(sizeof(T) * V + 3) / 4]; };
// the same value, but what was made of it before is made of it anew and not kept in registers until then
template <typename T, int V> __device__ __forceinline__ void afresh(Raw<T, V> &r)
{
#pragma unroll
    for (auto &w : r.w) asm volatile("" : "+v"(w));
}
// formed step by step: what all steps add, side by side until it is summed, would not fit the registers
__device__ __forceinline__ void here(int &e) { asm volatile("" : "+v"(e)); }
__device__ __forceinline__ void here(float &f) { asm volatile("" : "+v"(f)); }
template <typename T, int V, bool VEC> __device__ __forceinline__ Raw<T, V> fetch(const T *p, int left)
{
    Raw<T, V> r = {};
    if constexpr (VEC) {
        if (left > 0) __builtin_memcpy(&r, __builtin_assume_aligned(p, sizeof(T) * V), sizeof(T) * V);
    } else if (left >= V) {
        __builtin_memcpy(&r, p, sizeof(T) * V);
    } else if (left > 0) {
        T e[V];
#pragma unroll
        for (int v = 0; v < V; ++v) e[v] = v < left ? p[v] : (T)0.f;
        __builtin_memcpy(&r, e, sizeof(e));
    }
    return r;
}
template <typename T, int V> __device__ __forceinline__ float value(const Raw<T, V> &r, int v)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(r.w[v]);
    return __uint_as_float(v % 2 ? r.w[v / 2] & 0xffff0000u : r.w[v / 2] << 16);
}
template <typename T, int V, bool VEC> __device__ __forceinline__ void keep(T *p, const float (&f)[V], int left)
{
    T e[V];
#pragma unroll
    for (int v = 0; v < V; ++v) e[v] = (T)f[v];
    if constexpr (VEC) {
        if (left > 0) __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T) * V), e, sizeof(e));
    } else if (left >= V) {
        __builtin_memcpy(p, e, sizeof(e));
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v < left) p[v] = e[v];
    }
}

// words between workgroups
constexpr uint32_t kClear = 0xffffffffu;
__device__ __forceinline__ uint32_t told(float f)
{
    const uint32_t u = __float_as_uint(f);
    return u == kClear ? 0x7fc00000u : u;      // (a NaN all the same)
}
template <typename W> __device__ __forceinline__ void tell(W *p, W w) { __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename W> __device__ __forceinline__ W hear(const W *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

template <int V> using OutWord = std::conditional_t<V == 2, unsigned long long, uint32_t>;
struct Work {
    uint32_t *next;          // the counter that hands out tiles
    unsigned long long *span; // [tile][channel] m, H
    uint32_t *power;         // [tile][lane] e of its channels
    void *out;               // [tile][lane] what goes out of its channels, one word
};

// a call's kind: element type, channels a lane, whether these lie in whole words, direction, mix, and the gate's form
template <typename T_, int V_, bool VEC_, bool BACK_, bool MIX_, int FORM_> struct Kind {
    using T = T_;
    static constexpr int V = V_, FORM = FORM_;
    static constexpr bool VEC = VEC_, BACK = BACK_, MIX = MIX_;
};

// steps of a chain in the order of the recurrence: step s is token s, or of the backward token L - 1 - s
template <typename T, int V, bool VEC, bool BACK> struct Chain {
    const Gated &a;
    const T *x, *g, *dy, *yin;      // (of the wavefront's first channel: the same for all lanes)
    T *o0, *o1;
    const float *in;
    float *out;
    long long state;    // (of the first channel)
    int left;           // channels from this lane's first on
    unsigned mine;      // this lane's first
    __device__ __forceinline__ Chain(const Gated &a_, int chain, int groups, int lane) : a(a_)
    {
        const int sequence = __builtin_amdgcn_readfirstlane((unsigned)chain / (unsigned)groups);
        const long long b = sequence;
        const int c = (chain - sequence * groups) * (64 * V);
        mine = lane * V;
        left = a.D - c - (int)mine;
        const long long at = b * a.L * a.D + c;
        state = b * a.D + c;
        x = static_cast<const T *>(a.X) + (a.X ? b * a.xb + c : 0);
        g = static_cast<const T *>(a.G) + b * a.gb + c;
        if constexpr (BACK) {
            dy = static_cast<const T *>(a.dY) + b * a.dyb + c;
            yin = static_cast<const T *>(a.Yin) + at;
            o0 = static_cast<T *>(a.dX) + at;
            o1 = static_cast<T *>(a.dG) + at;
            in = a.dhL;
            out = a.dh0;
        } else {
            o0 = static_cast<T *>(a.Y) + at;
            in = a.h0;
            out = a.hL;
        }
    }
    __device__ __forceinline__ void incoming(float (&v)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = in && i < left ? in[state + mine + i] : 0.f;
    }
    __device__ __forceinline__ void outgoing(const float (&v)[V]) const
    {
        if (out)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < left) out[state + mine + i] = v[i];
    }
};

template <typename K, int N, bool KEPT, bool BACK = K::BACK> struct Span;

// Forward: N steps in registers.  Each is needed twice.  KEPT, with the mix, whose gates cost most: a and b stay in registers once they are
// formed (fp32: in the place of g and x; bf16: twice that, so fewer steps).  2 x 8192 x 4096 in bf16, 24 steps formed twice 118 us, 20 kept
// 106; 64 x 512 x 2048 96 and 90; 3 x 4099 x 1001 in fp32 51 and 47.  Without the mix they are formed twice.
template <typename K, int N, bool KEPT> struct Span<K, N, KEPT, false> {
    using T = typename K::T;
    static constexpr int V = K::V, FORM = K::FORM;
    static constexpr bool VEC = K::VEC, MIX = K::MIX;
    using C = Chain<T, V, VEC, false>;
    Raw<T, V> x[N], g[N];
    float a[KEPT ? N : 1][V], b[KEPT ? N : 1][V];
    __device__ __forceinline__ void read(const C &c, int s0)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const long long t = s0 + i;
            const int left = t < c.a.L ? c.left : 0;
            g[i] = fetch<T, V, VEC>(c.g + t * c.a.gt + c.mine, left);
            x[i] = fetch<T, V, VEC>(c.x + t * c.a.xt + c.mine, left);
        }
    }
    __device__ __forceinline__ void gates(const C &c, int s0, Product (&A)[V], float (&H)[V])
    {
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = {}, H[v] = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gate k = gate_of<FORM, MIX, sizeof(T) == 4>(value(g[i], v));
                const float in = MIX ? k.rest * value(x[i], v) : value(x[i], v), now = s0 + i < c.a.L ? k.a : 1.f;      // (behind the end x is zero)
                if constexpr (KEPT) a[i][v] = k.a, b[i][v] = in;
                A[v].times(now);
                H[v] = fmaf(now, H[v], in);
                here(A[v].e);
                if (v == V - 1 && i % 4 == 3) __builtin_amdgcn_sched_barrier(0);      // (all gates side by side would not fit the registers)
            }
#pragma unroll
        for (int v = 0; v < V; ++v) A[v].ready();
    }
    __device__ __forceinline__ void run(const C &c, int s0, float (&v)[V])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (s0 + i >= c.a.L) break;
            if constexpr (!KEPT) afresh(g[i]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if constexpr (KEPT) {
                    v[j] = fmaf(a[i][j], v[j], b[i][j]);
                } else {
                    const Gate k = gate_of<FORM, MIX, sizeof(T) == 4>(value(g[i], j));
                    v[j] = fmaf(k.a, v[j], MIX ? k.rest * value(x[i], j) : value(x[i], j));
                }
            }
            keep<T, V, VEC>(c.o0 + (long long)(s0 + i) * c.a.D + c.mine, v, c.left);
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
    }
};

template <typename K, int N, bool KEPT> struct Span<K, N, KEPT, true> {
    using T = typename K::T;
    static constexpr int V = K::V, FORM = K::FORM;
    static constexpr bool VEC = K::VEC, MIX = K::MIX;
    using C = Chain<T, V, VEC, true>;
    Raw<T, V> x[MIX ? N : 1], g[N], dy[N], y[N];
    __device__ __forceinline__ void read(const C &c, int s0)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const long long t = (long long)c.a.L - 1 - s0 - i;
            const int left = t >= 0 ? c.left : 0;
            g[i] = fetch<T, V, VEC>(c.g + t * c.a.gt + c.mine, left);
            dy[i] = fetch<T, V, VEC>(c.dy + t * c.a.dyt + c.mine, left);
            y[i] = fetch<T, V, VEC>(c.yin + (t - 1) * c.a.D + c.mine, t > 0 ? c.left : 0);
            if (MIX) x[MIX ? i : 0] = fetch<T, V, VEC>(c.x + t * c.a.xt + c.mine, left);
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);      // (the addresses of all rows would not fit the scalar registers)
        }
    }
    __device__ __forceinline__ void gates(const C &c, int s0, Product (&A)[V], float (&H)[V])
    {
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = {}, H[v] = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float a = s0 + i < c.a.L ? gate_of<FORM, false, sizeof(T) == 4>(value(g[i], v)).a : 1.f;
                A[v].times(a);
                H[v] = a * (value(dy[i], v) + H[v]);
                here(A[v].e);
                here(H[v]);
                if (v == V - 1 && i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
        for (int v = 0; v < V; ++v) A[v].ready();
    }
    __device__ __forceinline__ void run(const C &c, int s0, float (&v)[V])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const long long t = (long long)c.a.L - 1 - s0 - i;
            if (t < 0) break;
            afresh(g[i]);
            afresh(dy[i]);
            float dx[V], dg[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const Gate k = gate_of<FORM, MIX, sizeof(T) == 4>(value(g[i], j));
                const float l = value(dy[i], j) + v[j];
                float h = t > 0 ? value(y[i], j) : c.a.h0 && j < c.left ? c.a.h0[c.state + c.mine + j] : 0.f;
                if (MIX) h -= value(x[MIX ? i : 0], j);
                dx[j] = MIX ? k.rest * l : l;
                dg[j] = l * h * k.slope;
                v[j] = k.a * l;
            }
            keep<T, V, VEC>(c.o0 + t * c.a.D + c.mine, dx, c.left);
            keep<T, V, VEC>(c.o1 + t * c.a.D + c.mine, dg, c.left);
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
    }
};

struct Pair { float m, H; };
template <int V> struct WalkLds {
    Pair spans[2][kWaves][V][64];
    uint32_t powers[2][kWaves][64];
};

// A workgroup for each chain, from tile to tile.
template <typename K>
__device__ __forceinline__ void gated_walk(const Gated &a, int groups, WalkLds<K::V> &lds)
{
    using T = typename K::T;
    constexpr int V = K::V;
    constexpr bool VEC = K::VEC;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Chain<T, V, VEC, K::BACK> c(a, blockIdx.x, groups, lane);
    float in[V];
    c.incoming(in);
    Span<K, kWalkSteps, !K::BACK && K::MIX> s;
    for (int s0 = 0, turn = 0; s0 < a.L; s0 += kWaves * kWalkSteps, turn ^= 1) {
        const int mine = s0 + w * kWalkSteps;
        s.read(c, mine);
        Product A[V];
        float H[V];
        s.gates(c, mine, A, H);
#pragma unroll
        for (int v = 0; v < V; ++v) lds.spans[turn][w][v][lane] = {A[v].m, H[v]};
        lds.powers[turn][w][lane] = powers(A);
        __syncthreads();
        float now[V];
#pragma unroll 1
        for (int i = 0; i < kWaves; ++i) {
            const uint32_t e = lds.powers[turn][i][lane];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (i == w) now[v] = in[v];
                const Pair p = lds.spans[turn][i][v][lane];
                in[v] = through(p.m, power(e, v), p.H, in[v]);
            }
        }
        s.run(c, mine, now);
        if (s0 + kWaves * kWalkSteps >= a.L && w == kWaves - 1) c.outgoing(now);
    }
}

// A workgroup for each tile.
template <int V, int PER> struct TileLds {
    Pair spans[kWaves][V][64], behind[kWaves * PER][V][64];
    uint32_t powers[kWaves][64], behind_powers[kWaves * PER][64];
    float outs[kWaves * PER][V][64];
    int heard[kWaves * PER];      // of a tile in front: 1 its (A, H), 2 what goes out of it
    uint32_t ticket;
};
template <typename K, int PER>
__device__ __forceinline__ void gated_tile(const Gated &a, int groups, int chains, int tiles, const Work &work, TileLds<K::V, PER> &lds)
{
    using T = typename K::T;
    constexpr int V = K::V;
    constexpr bool VEC = K::VEC;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t id = __builtin_amdgcn_readfirstlane(lds.ticket);
    const int tile = __builtin_amdgcn_readfirstlane(id / chains), chain = (int)id - tile * chains;      // (unsigned division is done in the lanes)
    constexpr int steps = kTileSteps<T, K::BACK, K::MIX, (PER > 1)>;
    const int mine = (tile * kWaves + w) * steps;
    const Chain<T, V, VEC, K::BACK> c(a, chain, groups, lane);
    Span<K, steps, !K::BACK && K::MIX && (sizeof(T) == 4 || PER == 1)> s;
    s.read(c, mine);
    Product A[V];
    float H[V];
    s.gates(c, mine, A, H);
#pragma unroll
    for (int v = 0; v < V; ++v) lds.spans[w][v][lane] = {A[v].m, H[v]};
    lds.powers[w][lane] = powers(A);
    float in[V];
    if (tile == 0 && w == 0) {
        // read once, and there before anything of this tile is told: what goes out of the chain may be written in its place
        c.incoming(in);
#pragma unroll
        for (int v = 0; v < V; ++v) lds.outs[0][v][lane] = in[v];
    }
    __syncthreads();
    // words of a tile of this chain lie side by side: [tile][chain][v][lane]
    const long long row = (long long)chains * (64 * V), at = (long long)tile * row + (long long)chain * (64 * V);
    const long long power_row = (long long)chains * 64, power_at = (long long)tile * power_row + (long long)chain * 64;
    if (w == 0 && tile < tiles - 1) {
#pragma unroll 1
        for (int i = 1; i < kWaves; ++i) {
            const uint32_t e = lds.powers[i][lane];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Pair p = lds.spans[i][v][lane];
                H[v] = through(p.m, power(e, v), p.H, H[v]);
                A[v].times(p.m);
                A[v].e += power(e, v);
                A[v].ready();
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) A[v].e = min(max(A[v].e, -400), 400);      // (a power of 400 takes every state out of fp32)
        if (tile > 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) tell(work.span + at + 64 * v + (unsigned)lane, (unsigned long long)told(H[v]) << 32 | told(A[v].m));
            tell(work.power + power_at + (unsigned)lane, powers(A));
        }
    }
    if (tile == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = lds.outs[0][v][lane];
    } else {      // each wavefront listens to PER of the tiles in front
        bool has_out[PER] = {}, has_span[PER] = {};
        int from;
        while (true) {
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const int k = q * kWaves + w;
                const long long there = at - (long long)min(k + 1, tile) * row;
                if (!has_span[q] && k < tile - 1) {      // (the first tile only tells what goes out)
                    bool ready = true;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const unsigned long long p = hear(work.span + there + 64 * v + (unsigned)lane);
                        ready = ready && (uint32_t)p != kClear;
                        lds.behind[k][v][lane] = {__uint_as_float((uint32_t)p), __uint_as_float((uint32_t)(p >> 32))};
                    }
                    const uint32_t e = hear(work.power + power_at - (k + 1) * power_row + (unsigned)lane);
                    lds.behind_powers[k][lane] = e;
                    has_span[q] = __all(ready && e != kClear);
                }
                if (!has_out[q] && k < tile) {
                    const OutWord<V> o = hear(static_cast<const OutWord<V> *>(work.out) + (power_at - (k + 1) * power_row) + (unsigned)lane);
#pragma unroll
                    for (int v = 0; v < V; ++v) lds.outs[k][v][lane] = __uint_as_float((uint32_t)(v ? o >> 16 >> 16 : o));
                    has_out[q] = __all((uint32_t)o != kClear);
                }
                if (lane == 0) lds.heard[k] = (has_span[q] ? 1 : 0) | (has_out[q] ? 2 : 0);
            }
            __syncthreads();
            from = -1;      // the nearest tile whose outgoing values are told, if all between have told their (A, H)
            bool open = true;
#pragma unroll
            for (int k = 0; k < kWaves * PER; ++k) {
                const int h = lds.heard[k];
                if (open && (h & 2)) from = k, open = false;
                open = open && (h & 1);
            }
            from = __builtin_amdgcn_readfirstlane(from);
            if (from >= 0) break;
            __syncthreads();
        }
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = lds.outs[from][v][lane];
#pragma unroll 1
        for (int k = from - 1; k >= 0; --k) {
            const uint32_t e = lds.behind_powers[k][lane];
#pragma unroll
            for (int v = 0; v < V; ++v) in[v] = through(lds.behind[k][v][lane].m, power(e, v), lds.behind[k][v][lane].H, in[v]);
        }
    }
    if (w == 0 && tile < tiles - 1) {
        OutWord<V> o = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) o |= (OutWord<V>)told(through(A[v].m, A[v].e, H[v], in[v])) << (32 * v);
        tell(static_cast<OutWord<V> *>(work.out) + power_at + (unsigned)lane, o);
    }
#pragma unroll 1
    for (int i = 0; i < w; ++i) {
        const uint32_t e = lds.powers[i][lane];
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = through(lds.spans[i][v][lane].m, power(e, v), lds.spans[i][v][lane].H, in[v]);
    }
    s.run(c, mine, in);
    if (tile == tiles - 1 && w == kWaves - 1) c.outgoing(in);
}

__global__ __launch_bounds__(256) void gated_clear_kernel(u32x4 *p, long long n)
{
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) p[i] = kClear;
}

// A few steps: a lane takes V channels through all of them.
template <typename K>
__device__ __forceinline__ void gated_few(const Gated &a, int groups)
{
    using T = typename K::T;
    constexpr int V = K::V;
    constexpr bool VEC = K::VEC;
    const Chain<T, V, VEC, K::BACK> c(a, blockIdx.x, groups, threadIdx.x);
    float v[V];
    c.incoming(v);
    Span<K, 4, false> s;
    for (int s0 = 0; s0 < a.L; s0 += 4) {
        s.read(c, s0);
        s.run(c, s0, v);
    }
    c.outgoing(v);
}

// The gate's form is asked once, not at every step: a body for each.
template <typename T, int V, bool VEC, bool BACK, bool MIX, typename F> __device__ __forceinline__ void by_form(int gate, F f)
{
    if (gate == 0) f(Kind<T, V, VEC, BACK, MIX, 0>{});
    else if (gate == 1) f(Kind<T, V, VEC, BACK, MIX, 1>{});
    else f(Kind<T, V, VEC, BACK, MIX, 2>{});
}
template <typename T, int V, bool VEC, bool BACK, bool MIX>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(4))) void gated_walk_kernel(Gated a, int groups)
{
    __shared__ WalkLds<V> lds;
    by_form<T, V, VEC, BACK, MIX>(a.gate, [&](auto k) { gated_walk<decltype(k)>(a, groups, lds); });
}
// (so many wavefronts to a SIMD; where channels lie at odd places their registers allow three)
template <typename T, int V, bool VEC, bool BACK, bool MIX, int PER>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(!VEC ? 3 : BACK && PER == 1 ? 6 : 4)))
void gated_tile_kernel(Gated a, int groups, int chains, int tiles, Work work)
{
    __shared__ TileLds<V, PER> lds;
    if (threadIdx.x == 0) lds.ticket = __hip_atomic_fetch_add(work.next, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u;
    __syncthreads();
    by_form<T, V, VEC, BACK, MIX>(a.gate, [&](auto k) { gated_tile<decltype(k), PER>(a, groups, chains, tiles, work, lds); });
}
template <typename T, int V, bool VEC, bool BACK, bool MIX> __global__ __launch_bounds__(64) void gated_few_kernel(Gated a, int groups)
{
    by_form<T, V, VEC, BACK, MIX>(a.gate, [&](auto k) { gated_few<decltype(k)>(a, groups); });
}

enum { kFew, kWalk, kTiles };
struct Plan {
    int how, groups, chains, tiles;
    bool farther;
    size_t bytes;
};
Plan plan(int B, int L, int D, bool is_bf16, bool back, bool mix)
{
    const int V = is_bf16 ? 2 : 1;
    Plan p = {};
    p.groups = (int)((D + 64LL * V - 1) / (64 * V));
    p.chains = (int)std::min((long long)B * p.groups, (long long)INT_MAX);      // (launch refuses as many)
    // Few chains have many of their tiles on the chip at once: listening to sixteen, and backward tiles of 16 steps, two workgroups to a
    // compute unit, make a long sequence's chain shorter: 1 x 65536 in bf16, forward 64 channels 69 -> 64 us, 512: 83 -> 76, 1024: 104 -> 116;
    // backward 64: 174 -> 87, 512: 193 -> 109, 1024: 215 -> 182, 1 x 16384 x 512 64 -> 43; where tiles are few, 1 x 3000 x 512 with the mix, 20 -> 22.
    p.farther = p.chains <= (back ? 8 : 6);
    auto tiles = [&] {
        const int tile = back ? tile_tokens<bf16, true, false>(p.farther) : !is_bf16 ? tile_tokens<float, false, false>(p.farther)
                         : mix ? tile_tokens<bf16, false, true>(p.farther) : tile_tokens<bf16, false, false>(p.farther);
        p.tiles = L / tile + (L % tile != 0);
    };
    tiles();
    if (p.farther && p.tiles <= 8 * kWaves) p.farther = false, tiles();
    p.how = L <= 16 ? kFew : L <= 2 * kWaves * kWalkSteps || p.chains >= 4 * device_cu_count() ? kWalk : kTiles;
    if (p.how == kTiles) p.bytes = 256 + (size_t)p.tiles * p.chains * 64 * (12 * V + 4);
    return p;
}

template <bool BACK> hipError_t launch(const Gated &a, bool is_bf16, bool aligned, hipStream_t stream)
{
    const Plan p = plan(a.B, a.L, a.D, is_bf16, BACK, a.mix);
    const double chains = (double)a.B * p.groups;
    if (!launch_holds(p.how == kTiles ? chains * p.tiles : chains, p.how == kFew ? 64 : 64 * kWaves)) return hipErrorInvalidConfiguration;
    auto with_mix = [&](auto one, auto vec, auto mix) {
        using T = decltype(one);
        constexpr int V = sizeof(T) == 2 ? 2 : 1;
        if (p.how == kFew) {
            hipLaunchKernelGGL((gated_few_kernel<T, V, vec.value, BACK, mix.value>), dim3(p.chains), dim3(64), 0, stream, a, p.groups);
        } else if (p.how == kWalk) {
            hipLaunchKernelGGL((gated_walk_kernel<T, V, vec.value, BACK, mix.value>), dim3(p.chains), dim3(64 * kWaves), 0, stream, a, p.groups);
        } else {
            const long long n = (long long)((p.bytes + 15) / 16), blocks = (n + 255) / 256, most = 8LL * device_cu_count();
            hipLaunchKernelGGL(gated_clear_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, stream,
                               static_cast<u32x4 *>(a.work), n);
            const size_t words = (size_t)p.tiles * p.chains * (64 * V);
            char *base = static_cast<char *>(a.work);
            Work work;
            work.next = reinterpret_cast<uint32_t *>(base);
            work.span = reinterpret_cast<unsigned long long *>(base + 256);
            work.out = base + 256 + words * 8;
            work.power = reinterpret_cast<uint32_t *>(base + 256 + words * 12);
            const long long count = (long long)p.chains * p.tiles;
            auto kernel = p.farther ? gated_tile_kernel<T, V, vec.value, BACK, mix.value, 2>
                                    : gated_tile_kernel<T, V, vec.value, BACK, mix.value, 1>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(64 * kWaves), 0, stream, a, p.groups, p.chains, p.tiles, work);
        }
    };
    auto with = [&](auto one, auto vec) {
        if (a.mix) with_mix(one, vec, std::true_type{});
        else with_mix(one, vec, std::false_type{});
    };
    if (is_bf16) {
        if (aligned) with((bf16)0.f, std::true_type{});
        else with((bf16)0.f, std::false_type{});
    } else {
        with(0.f, std::true_type{});
    }
    return hipGetLastError();
}

// whether V channels of a token lie in whole words everywhere (fp32 takes one at a time)
inline bool words(const void *p, long long batch, long long token)
{
    return reinterpret_cast<uintptr_t>(p) % 4 == 0 && batch % 2 == 0 && token % 2 == 0;
}

}  // namespace

size_t gated_workspace_bytes(int B, int L, int D, bool is_bf16)
{
    const size_t n = std::max({plan(B, L, D, is_bf16, false, false).bytes, plan(B, L, D, is_bf16, false, true).bytes,
                               plan(B, L, D, is_bf16, true, false).bytes});
    return (n + 15) / 16 * 16;
}

hipError_t launch_gated_fwd(const Gated &a, bool is_bf16, hipStream_t stream)
{
    return launch<false>(a, is_bf16, a.D % 2 == 0 && words(a.X, a.xb, a.xt) && words(a.G, a.gb, a.gt), stream);
}

hipError_t launch_gated_bwd(const Gated &a, bool is_bf16, hipStream_t stream)
{
    return launch<true>(a, is_bf16, a.D % 2 == 0 && (!a.X || words(a.X, a.xb, a.xt)) && words(a.G, a.gb, a.gt) && words(a.dY, a.dyb, a.dyt),
                        stream);
}

}  // namespace pf
