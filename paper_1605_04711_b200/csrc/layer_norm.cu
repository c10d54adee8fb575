// Layer norm over the channels of a row (a token, or a pixel of an NHWC tensor), forward and backward.
//
//   forward   mean = sum x / C,  var = sum (x - mean)^2 / C,  rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd gamma + beta
//   backward  xh = (x - mean) rstd,  g = dy gamma,  dx = rstd (g - sum(g) / C - xh sum(g xh) / C),
//             dgamma = sum over the rows of dy xh,  dbeta = sum over the rows of dy
//   computed with d = x - mean and h = rstd g, so that xh is never formed:  dx = h - sum(h) / C - d rstd^2 sum(h d) / C
//
// Both are bound by HBM: a row is read once and stays in registers until its result is written.  A team of T threads (4 to
// 1024, a power of two) has a row, E elements a thread; its sums are shuffle trees, and one barrier where it is more than a
// warp.  The variance is that of the differences from the mean (a second tree), never a difference of two sums: rows far from
// zero keep their digits.  All arithmetic is fp32, rounded once to the type of the output.
#include <algorithm>
#include <cmath>

#include <cuda_bf16.h>

#include "common.cuh"
#include "tc_ptx.cuh"

namespace {

using bf16 = __nv_bfloat16;

// V consecutive elements in one or two 16-byte accesses, or one element where rows or bases are not aligned.
template <typename T, int V> struct Vec;
template <> struct Vec<bf16, 8> {
    uint4 r;
    __device__ void load(const bf16 *p) { r = *reinterpret_cast<const uint4 *>(p); }
    __device__ void zero() { r = make_uint4(0u, 0u, 0u, 0u); }
    __device__ void get(float (&f)[8]) const
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
};
template <> struct Vec<bf16, 4> {
    uint2 r;
    __device__ void load(const bf16 *p) { r = *reinterpret_cast<const uint2 *>(p); }
    __device__ void zero() { r = make_uint2(0u, 0u); }
    __device__ void get(float (&f)[4]) const
    {
        f[0] = __uint_as_float(r.x << 16); f[1] = __uint_as_float(r.x & 0xFFFF0000u);
        f[2] = __uint_as_float(r.y << 16); f[3] = __uint_as_float(r.y & 0xFFFF0000u);
    }
};
template <> struct Vec<float, 4> {
    float4 r;
    __device__ void load(const float *p) { r = *reinterpret_cast<const float4 *>(p); }
    __device__ void zero() { r = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ void get(float (&f)[4]) const { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
};
template <> struct Vec<float, 8> {
    float4 r[2];
    __device__ void load(const float *p)
    {
        r[0] = *reinterpret_cast<const float4 *>(p);
        r[1] = *reinterpret_cast<const float4 *>(p + 4);
    }
    __device__ void zero() { r[0] = r[1] = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ void get(float (&f)[8]) const
    {
        f[0] = r[0].x; f[1] = r[0].y; f[2] = r[0].z; f[3] = r[0].w;
        f[4] = r[1].x; f[5] = r[1].y; f[6] = r[1].z; f[7] = r[1].w;
    }
};
template <typename T> struct Vec<T, 1> {
    T r;
    __device__ void load(const T *p) { r = *p; }
    __device__ void zero() { r = T(0.0f); }
    __device__ void get(float (&f)[1]) const { f[0] = (float)r; }
};

__device__ __forceinline__ uint32_t two_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ void store(bf16 *p, const float (&f)[8])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(two_bf16(f[0], f[1]), two_bf16(f[2], f[3]), two_bf16(f[4], f[5]), two_bf16(f[6], f[7]));
}
__device__ __forceinline__ void store(bf16 *p, const float (&f)[4])
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(two_bf16(f[0], f[1]), two_bf16(f[2], f[3]));
}
__device__ __forceinline__ void store(bf16 *p, const float (&f)[1]) { *p = __float2bfloat16_rn(f[0]); }
__device__ __forceinline__ void store(float *p, const float (&f)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store(float *p, const float (&f)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]); }
__device__ __forceinline__ void store(float *p, const float (&f)[1]) { *p = f[0]; }

// gamma and beta: fp32, `none` where the caller has none.  Loads of read-only data, which the compiler may take ahead of the
// stores of earlier columns.
template <int V> __device__ __forceinline__ void load_param(float (&f)[V], const float *p, long long col, float none)
{
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = none;
    } else if constexpr (V == 1) {
        f[0] = __ldg(p + col);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 v = __ldg(reinterpret_cast<const float4 *>(p + col + i));
            f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
        }
    }
}

// Two fp32 numbers in one register pair: Blackwell adds, multiplies and fuses both in one instruction.
typedef unsigned long long two_f32;
__device__ __forceinline__ two_f32 two(float a, float b)
{
    two_f32 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void each(two_f32 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ two_f32 add2(two_f32 a, two_f32 b)
{
    two_f32 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ two_f32 mul2(two_f32 a, two_f32 b)
{
    two_f32 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ two_f32 fma2(two_f32 a, two_f32 b, two_f32 c)
{
    two_f32 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float sum2(two_f32 v)
{
    float a, b;
    each(v, a, b);
    return a + b;
}

// Sums over a team of T threads, the same bits in all of them.  Every thread of the team calls it (and of the warp, where that
// has several teams).  `red` holds two floats for each of 32 warps, twice: a buffer is written again one barrier after all
// have read it.  `barrier`: the team's own, 0 for a block that is one team.
template <int N> __device__ __forceinline__ void team_sum(float (&v)[N], int T, float (*red)[32][2], unsigned int &turn, int barrier)
{
    const int span = min(T, 32);
    for (int o = span >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (T > 32) {
        float(*buf)[2] = red[turn & 1];
        ++turn;
        const int warp = threadIdx.x >> 5, warps = T >> 5, first = warp / warps * warps;
        if ((threadIdx.x & 31) == 0) *reinterpret_cast<float2 *>(buf[warp]) = make_float2(v[0], N > 1 ? v[N - 1] : 0.0f);
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(T) : "memory");
        v[0] = v[N - 1] = 0.0f;
#pragma unroll 4
        for (int w = first; w < first + warps; ++w) {
            const float2 a = *reinterpret_cast<const float2 *>(buf[w]);
            v[0] += a.x;
            if (N > 1) v[N - 1] += a.y;
        }
    }
}

// The same for a team whose size is known at compile time.  Two sums share their shuffles: of a pair of lanes each goes on with one.
template <int TT, int N> __device__ __forceinline__ void team_sum(float (&v)[N], float (*red)[32][2], unsigned int &turn, int barrier)
{
    constexpr int kSpan = TT < 32 ? TT : 32, kWarps = TT / 32;
    const int lane = threadIdx.x & 31;
    float own = v[0];
    if (N == 2) {
        const bool odd = lane & 1;
        own = (odd ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, odd ? v[0] : v[1], 1);
    }
#pragma unroll
    for (int o = N; o < kSpan; o <<= 1) own += __shfl_xor_sync(0xffffffffu, own, o);
    if (TT <= 32) {
        if (N == 1) {
            v[0] = own;
        } else {
            const float other = __shfl_xor_sync(0xffffffffu, own, 1);
            v[0] = lane & 1 ? other : own;
            v[N - 1] = lane & 1 ? own : other;
        }
    } else {
        // a warp's sums, its one or two floats next to the next warp's
        float *const buf = &red[turn & 1][0][0];
        ++turn;
        const int warp = threadIdx.x >> 5, first = warp / (kWarps ? kWarps : 1) * kWarps;
        if (lane < N) buf[warp * N + lane] = own;
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(TT) : "memory");
        if (N == 2) {
            two_f32 s = 0;
#pragma unroll
            for (int w = 0; w < kWarps; w += 2) {
                const float4 a = *reinterpret_cast<const float4 *>(buf + (first + w) * 2);
                s = add2(add2(s, two(a.x, a.y)), two(a.z, a.w));
            }
            each(s, v[0], v[N - 1]);
        } else {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; w += 2) {
                const float2 a = *reinterpret_cast<const float2 *>(buf + first + w);
                s += a.x + a.y;
            }
            v[0] = s;
        }
    }
}

// Column of a thread's vector j, and whether the vectors j of the whole team lie inside the row (the same for all threads).  TT: the
// team's size where it is known at compile time, so that single elements (V = 1) lie at constant offsets of one address; with
// the offsets worked out for each, a row of 1001 took 85 instructions an element.
template <int V, int TT> struct Columns {
    int T_, t, C;
    __device__ __forceinline__ int T() const { return TT ? TT : T_; }
    __device__ __forceinline__ int operator()(int j) const { return (j * T() + t) * V; }
    __device__ __forceinline__ bool whole(int j) const { return (j + 1) * T() * V <= C; }
};
// N vectors from j on into raw, nothing past the row's end.
template <typename T, int V, int TT, int N> __device__ __forceinline__ void load_vectors(Vec<T, V> (&raw)[N], const T *row, const Columns<V, TT> &col, bool live)
{
    constexpr int K = N < 8 ? N : 8;
#pragma unroll
    for (int j0 = 0; j0 < N; j0 += K) {
        if (live && col.whole(j0 + K - 1)) {
#pragma unroll
            for (int j = j0; j < j0 + K; ++j) raw[j].load(row + col(j));
        } else {
#pragma unroll
            for (int j = j0; j < j0 + K; ++j)
                if (live && col(j) < col.C) raw[j].load(row + col(j));
                else raw[j].zero();
        }
    }
}
template <typename T, int V, int TT> __device__ __forceinline__ void read_vector(const T *row, const Columns<V, TT> &col, int j, float (&f)[V])
{
    Vec<T, V> v;
    if (col.whole(j)) {
        v.load(row + col(j));
    } else if (col(j) < col.C) {
        v.load(row + col(j));
    } else {
        v.zero();
    }
    v.get(f);
}

template <typename T, int V, int TT> __device__ __forceinline__ void add_vector(float (&f)[V], const T *row, const Columns<V, TT> &col, int j)
{
    float e[V];
    read_vector(row, col, j, e);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] += e[i];
}

struct FwdParams {
    const void *X;
    void *Y;
    const float *gamma, *beta;
    float *mean, *rstd;
    long long ldx, ldy, M, C;
    float eps;
    int T;
};

// One row per team, in registers.  C <= T * E.  A team of more than a warp is a block.
template <typename TX, typename TY, int V, int E, int TT>
__global__ void __launch_bounds__(TT > 32 ? TT : TT == 32 || E < 16 ? 128 : 1024, TT <= 32 || V == 1 ? 1 : 1024 / (TT ? TT : 1)) norm_fwd_kernel(const __grid_constant__ FwdParams P)
{
    constexpr int NV = E / V, P2 = E / 2;
    __shared__ __align__(16) float red[2][32][2];
    unsigned int turn = 0;
    const int T = TT ? TT : P.T, t = threadIdx.x & (T - 1), C = (int)P.C;
    const int teams = blockDim.x / T, team = threadIdx.x / T;
    const float inv = 1.0f / (float)C;
    const Columns<V, TT> col{T, t, C};
    pdl_begin();
    for (long long r0 = (long long)blockIdx.x * teams; r0 < P.M; r0 += (long long)gridDim.x * teams) {
        const long long r = r0 + team;
        const bool live = r < P.M;
        const TX *x = static_cast<const TX *>(P.X) + (live ? r : 0) * P.ldx;
        Vec<TX, V> raw[NV];
        load_vectors(raw, x, col, live);
        two_f32 d[P2], s2 = 0, q2 = 0;
        {
            float f[E];
#pragma unroll
            for (int j = 0; j < NV; ++j) raw[j].get(*reinterpret_cast<float(*)[V]>(f + j * V));
#pragma unroll
            for (int i = 0; i < P2; ++i) {
                d[i] = two(f[2 * i], f[2 * i + 1]);
                s2 = add2(s2, d[i]);
            }
        }
        float s[1] = {sum2(s2)};
        if constexpr (TT > 0) team_sum<TT>(s, red, turn, 0);
        else team_sum(s, T, red, turn, 0);
        const float mean = s[0] * inv;
        const two_f32 minus = two(-mean, -mean);
#pragma unroll
        for (int i = 0; i < P2; ++i) d[i] = add2(d[i], minus);
        // nothing of what is past the row's end
        constexpr int K = NV < 8 ? NV : 8;
#pragma unroll
        for (int j0 = 0; j0 < NV; j0 += K)
            if (!col.whole(j0 + K - 1))
#pragma unroll
                for (int i = j0 * V / 2; i < (j0 + K) * V / 2; ++i) {
                    if (V > 1) {
                        if (col(2 * i / V) >= C) d[i] = 0;
                    } else {
                        float a, b;
                        each(d[i], a, b);
                        d[i] = two(col(2 * i) < C ? a : 0.0f, col(2 * i + 1) < C ? b : 0.0f);
                    }
                }
#pragma unroll
        for (int i = 0; i < P2; ++i) q2 = fma2(d[i], d[i], q2);
        float q[1] = {sum2(q2)};
        if constexpr (TT > 0) team_sum<TT>(q, red, turn, 0);
        else team_sum(q, T, red, turn, 0);
        const float rstd = rsqrtf(fmaf(q[0], inv, P.eps));
        if (!live) continue;
        const two_f32 scale = two(rstd, rstd);
        TY *y = static_cast<TY *>(P.Y) + r * P.ldy;
        // K vectors: whole where the team's are, so that their loads of gamma and beta go together
        auto put = [&](int j, const float(&ga)[V], const float(&be)[V]) {
            float o[V];
            if constexpr (V > 1) {
#pragma unroll
                for (int i = 0; i < V / 2; ++i)
                    each(fma2(mul2(d[j * V / 2 + i], scale), two(ga[2 * i], ga[2 * i + 1]), two(be[2 * i], be[2 * i + 1])), o[2 * i], o[2 * i + 1]);
            } else {
                float a, b;
                each(d[j / 2], a, b);
                o[0] = fmaf((j & 1 ? b : a) * rstd, ga[0], be[0]);
            }
            store(y + col(j), o);
        };
#pragma unroll
        for (int j0 = 0; j0 < NV; j0 += K) {
            const bool whole = col.whole(j0 + K - 1);
            if (whole && V == 1) {
                float ga[K][V], be[K][V];
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    load_param(ga[j], P.gamma, col(j0 + j), 1.0f);
                    load_param(be[j], P.beta, col(j0 + j), 0.0f);
                }
#pragma unroll
                for (int j = 0; j < K; ++j) put(j0 + j, ga[j], be[j]);
            } else {
#pragma unroll
                for (int j = j0; j < j0 + K; ++j) {
                    if (!whole && col(j) >= C) continue;
                    float ga[V], be[V];
                    load_param(ga, P.gamma, col(j), 1.0f);
                    load_param(be, P.beta, col(j), 0.0f);
                    put(j, ga, be);
                }
            }
        }
        if (t == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
    }
}

// ---- rows through shared memory ---------------------------------------------------------------------------------------------
// Large tensors of aligned rows.  With 16 elements a thread, all of them in registers, a row of 4096 took 31 instructions an element,
// most of them the fixed part of a row: two sums, the barriers, the root, the addresses; with more, few rows fit the registers, and
// too little is on its way.  Here rows come by bulk copies into a ring in shared memory, up to 192 KB an SM on their way, for threads
// of up to 64 elements.
constexpr int kMaxRing = 8, kMaxTeams = 32;
// Of the 227 KB that a block may have; 2.6 KB are barriers and sums.  Forward with 200 KB, two stages at 16384 x 4096 instead of three, took 48.0 us for 46.6;
// backward with 224 KB, three instead of two, 85.7 for 82.2.
constexpr size_t kFwdRingBytes = 224 * 1024, kBwdRingBytes = 200 * 1024;
struct Ring {
    int stages, stage_bytes, second;         // of a stage: where a second tensor's row begins
    int params;                              // bytes at the front that hold gamma (and beta), 0: they are read from global memory
};

// gamma or beta in shared memory: as it is, but for V = 8 the lower and the upper halves of eight apart, so that a warp's 16-byte
// reads are next to each other.
template <int V> __device__ __forceinline__ int param_at(int c, int C) { return V == 8 ? (c & 4 ? C / 2 : 0) + (c >> 3) * 4 + (c & 3) : c; }
template <int V> __device__ __forceinline__ void read_param(const float *sm, const float *global, int c, int C, float none, float (&f)[V])
{
    if (sm == nullptr) {
        load_param(f, global, c, none);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(sm + param_at<V>(c + i, C));
            f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
        }
    }
}

template <int E> constexpr int fwd_ring_threads() { return E >= 64 ? 512 : E >= 32 ? 768 : 1024; }

// TT > 0: teams of TT threads whose elements the row fills, C = TT E, so that addresses are constants and nothing is checked.
template <typename TX, typename TY, int V, int E, int TT>
__global__ void __launch_bounds__(fwd_ring_threads<E>(), 1) norm_fwd_ring_kernel(const __grid_constant__ FwdParams P, const __grid_constant__ Ring R)
{
    constexpr int NV = E / V, P2 = E / 2;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ unsigned long long full[kMaxTeams][kMaxRing];
    __shared__ __align__(16) float red[2][32][2];
    __shared__ volatile int gave_up;
    unsigned int turn = 0;
    const int T = TT ? TT : P.T, team = threadIdx.x / T, t = threadIdx.x - team * T, C = TT ? TT * E : (int)P.C;
    const int teams = blockDim.x / T, barrier = teams > 1 ? team + 1 : 0;
    const float inv = 1.0f / (float)C;
    const Columns<V, TT> col{T, t, C};
    if (t == 0)
        for (int s = 0; s < R.stages; ++s) mbar_init(&full[team][s], 1);
    if (threadIdx.x == 0) gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    pdl_begin();
    uint8_t *const mine = ring + R.params + (size_t)team * R.stages * R.stage_bytes;
    const long long first = (long long)blockIdx.x * teams + team, step = (long long)gridDim.x * teams;
    auto issue = [&](long long r, int s) {
        if (r >= P.M) return;
        mbar_expect_tx(&full[team][s], C * (uint32_t)sizeof(TX));
        bulk_load(mine + (size_t)s * R.stage_bytes, static_cast<const TX *>(P.X) + r * P.ldx, C * (uint32_t)sizeof(TX), &full[team][s]);
    };
    if (t == 0)
        for (int s = 0; s < R.stages; ++s) issue(first + s * step, s);
    const bool in_ring = TT ? 2 * TT * E * sizeof(float) <= kFwdRingBytes / 2 : R.params > 0;
    float *const gammas = in_ring ? reinterpret_cast<float *>(ring) : nullptr, *const betas = in_ring ? gammas + C : nullptr;
    if (in_ring) {
        for (int c = threadIdx.x; c < C; c += blockDim.x) {
            gammas[param_at<V>(c, C)] = P.gamma ? P.gamma[c] : 1.0f;
            betas[param_at<V>(c, C)] = P.beta ? P.beta[c] : 0.0f;
        }
        __syncthreads();
    }
    int s = 0;
    uint32_t ph = 0;
    for (long long r = first; r < P.M; r += step) {
        // a wait that ran out is no row: its results are NaNs
        const bool ok = mbar_wait(&full[team][s], ph, &gave_up, nullptr, 0);
        const TX *const row = reinterpret_cast<const TX *>(mine + (size_t)s * R.stage_bytes);
        two_f32 d[P2], s2 = 0, q2 = 0;
        {
            float f[E];
#pragma unroll
            for (int j = 0; j < NV; ++j) read_vector(row, col, j, *reinterpret_cast<float(*)[V]>(f + j * V));
#pragma unroll
            for (int i = 0; i < P2; ++i) {
                d[i] = two(f[2 * i], f[2 * i + 1]);
                s2 = add2(s2, d[i]);
            }
        }
        float sum[1] = {ok ? sum2(s2) : __uint_as_float(0x7FC00000u)};
        if constexpr (TT > 0) team_sum<TT>(sum, red, turn, barrier);
        else team_sum(sum, T, red, turn, barrier);
        // the whole team has its elements: the stage is free
        if (T == 32) __syncwarp();
        if (t == 0) issue(r + R.stages * step, s);
        const float mean = sum[0] * inv;
        const two_f32 minus = two(-mean, -mean);
#pragma unroll
        for (int i = 0; i < P2; ++i) {
            d[i] = add2(d[i], minus);
            // nothing of what is past the row's end
            if (!col.whole(2 * i / V) && col(2 * i / V) >= C) d[i] = 0;
            q2 = fma2(d[i], d[i], q2);
        }
        float q[1] = {sum2(q2)};
        if constexpr (TT > 0) team_sum<TT>(q, red, turn, barrier);
        else team_sum(q, T, red, turn, barrier);
        const float rstd = rsqrtf(fmaf(q[0], inv, P.eps));
        const two_f32 scale = two(rstd, rstd);
        TY *y = static_cast<TY *>(P.Y) + r * P.ldy;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!col.whole(j) && col(j) >= C) continue;
            float ga[V], be[V], o[V];
            read_param<V>(gammas, P.gamma, col(j), C, 1.0f, ga);
            read_param<V>(betas, P.beta, col(j), C, 0.0f, be);
#pragma unroll
            for (int i = 0; i < V / 2; ++i)
                each(fma2(mul2(d[j * V / 2 + i], scale), two(ga[2 * i], ga[2 * i + 1]), two(be[2 * i], be[2 * i + 1])), o[2 * i], o[2 * i + 1]);
            store(y + col(j), o);
        }
        if (t == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
        if (++s == R.stages) { s = 0; ph ^= 1u; }
    }
}

// Rows longer than the registers of a block: the row is read three times, from L2 after the first.
template <typename TX, typename TY, int V>
__global__ void __launch_bounds__(1024) norm_fwd_long_kernel(const __grid_constant__ FwdParams P)
{
    __shared__ __align__(16) float red[2][32][2];
    unsigned int turn = 0;
    const float inv = 1.0f / (float)P.C;
    pdl_begin();
    for (long long r = blockIdx.x; r < P.M; r += gridDim.x) {
        const TX *x = static_cast<const TX *>(P.X) + r * P.ldx;
        float s[1] = {0.0f}, f[V];
        for (long long col = (long long)threadIdx.x * V; col < P.C; col += 1024 * V) {
            Vec<TX, V> v;
            v.load(x + col);
            v.get(f);
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += f[i];
        }
        team_sum(s, 1024, red, turn, 0);
        const float mean = s[0] * inv;
        float q[1] = {0.0f};
        for (long long col = (long long)threadIdx.x * V; col < P.C; col += 1024 * V) {
            Vec<TX, V> v;
            v.load(x + col);
            v.get(f);
#pragma unroll
            for (int i = 0; i < V; ++i) q[0] = fmaf(f[i] - mean, f[i] - mean, q[0]);
        }
        team_sum(q, 1024, red, turn, 0);
        const float rstd = rsqrtf(fmaf(q[0], inv, P.eps));
        TY *y = static_cast<TY *>(P.Y) + r * P.ldy;
        for (long long col = (long long)threadIdx.x * V; col < P.C; col += 1024 * V) {
            Vec<TX, V> v;
            float ga[V], be[V];
            v.load(x + col);
            v.get(f);
            load_param(ga, P.gamma, col, 1.0f);
            load_param(be, P.beta, col, 0.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) ga[i] = fmaf((f[i] - mean) * rstd, ga[i], be[i]);
            store(y + col, ga);
        }
        if (threadIdx.x == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
    }
}

struct BwdParams {
    const void *dY, *X;
    void *dX;
    const void *add;             // added to dX
    const float *gamma, *mean, *rstd;
    float *part;                 // [parts][2][C]: sums of dy xh, sums of dy; NULL where the caller wants neither
    float *row_sums;             // long rows: [M][2]
    long long lddy, ldx, lddx, M, C;
    int T, parts;
    bool bulk;                   // rows of dY and X on 16-byte boundaries, a multiple of that long
};

constexpr int kBwdThreads = 512;

// The column sums of a block's `parties` (teams, or warps of several teams), of which this thread belongs to number `me`, to `out`, [2][C]; they are added in
// their order.  cols: [parties][2][C] in shared memory where there are several (with one after the other adding to one [2][C], the sixteen
// warps of a block took 5 of 29 us for rows of 64).
template <int V, int E, typename Col>
__device__ __forceinline__ void join_sums(const float (&g)[E], const float (&b)[E], const Col &col, bool mine, int me, int parties, float *cols, float *out)
{
    const int C = col.C;
    float *const to = parties > 1 ? cols + (size_t)me * 2 * C : out;
    if (mine)
#pragma unroll
        for (int j = 0; j < E / V; ++j) {
            if (col(j) >= C) continue;
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = g[j * V + i];
            store(to + col(j), v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = b[j * V + i];
            store(to + C + col(j), v);
        }
    if (parties == 1) return;
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * C; c += blockDim.x) {
        float v = 0.0f;
#pragma unroll 4
        for (int k = 0; k < parties; ++k) v += cols[(size_t)k * 2 * C + c];
        out[c] = v;
    }
}

// 16, 8 or 4 bytes to shared memory on their own way; zeros where `there` is false.
template <int BYTES> __device__ __forceinline__ void copy_piece(uint32_t dst, const void *src, bool there)
{
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(there ? BYTES : 0) : "memory");
}
// Bytes of a thread's part of a row in a stage: dY, X, mean and rstd.
template <typename TD, typename TX, int E> __host__ __device__ constexpr int bwd_stage_bytes() { return E * (int)(sizeof(TD) + sizeof(TX)) + 8; }
// A thread has sixteen elements of a row.  As many stages as fit 208 KB of shared memory for 512 threads: five where dY and X are bf16, three where both are fp32.
template <typename TD, typename TX> __host__ __device__ constexpr int bwd_stages() { return sizeof(TD) + sizeof(TX) == 4 ? 5 : sizeof(TD) + sizeof(TX) == 6 ? 4 : 3; }

// One row per team; sums over the rows of a block stay in the registers of the threads that own the columns, and its teams join them in
// shared memory at the end.  C <= T * E.  Vectors come through shared memory, every thread's own elements by its own copies, so no
// barrier guards them: two to four rows of every team are on their way.  Single elements (V = 1) of the next row are in registers.
// With sixteen elements a thread the fixed part of a row is half that of eight (32 M elements in rows of 2304, fp32: 83 us, 130 with eight).
template <typename TD, typename TX, typename TO, int V, int E, int TT>
__global__ void __launch_bounds__(kBwdThreads, 1) norm_bwd_kernel(const __grid_constant__ BwdParams P)
{
    constexpr int NV = E / V, P2 = E / 2;
    constexpr bool kRing = V > 1;
    constexpr uint32_t kStages = bwd_stages<TD, TX>();
    extern __shared__ __align__(16) uint8_t bwd_smem[];      // the stages; [2][C] sums when a block has several teams (of a warp or more)
    __shared__ __align__(16) float red[2][32][2];
    unsigned int turn = 0;
    const int T = TT ? TT : P.T, t = threadIdx.x & (T - 1), C = (int)P.C;
    const int teams = blockDim.x / T, team = threadIdx.x / T;
    const int barrier = teams > 1 ? team + 1 : 0;
    const float inv = 1.0f / (float)C;
    const long long step = (long long)gridDim.x * teams;
    const Columns<V, TT> col{T, t, C};
    pdl_begin();
    two_f32 ga[P2], a_g[P2], a_b[P2];
    {
        float f[E];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float g[V];
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = 0.0f;
            if (col(j) < C) load_param(g, P.gamma, col(j), 1.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[j * V + i] = g[i];
        }
#pragma unroll
        for (int i = 0; i < P2; ++i) { ga[i] = two(f[2 * i], f[2 * i + 1]); a_g[i] = a_b[i] = 0; }
    }
    Vec<TD, V> nd[NV];
    Vec<TX, V> nx[NV];
    float n_mean, n_rstd;
    auto fetch = [&](long long r) {
        const bool live = r < P.M;
        const TD *d = static_cast<const TD *>(P.dY) + (live ? r : 0) * P.lddy;
        const TX *x = static_cast<const TX *>(P.X) + (live ? r : 0) * P.ldx;
        n_mean = live ? P.mean[r] : 0.0f;
        n_rstd = live ? P.rstd[r] : 0.0f;
        load_vectors(nd, d, col, live);
        load_vectors(nx, x, col, live);
    };
    // a stage: vector j of dY of all threads, one next to the other, for every j; X likewise; the means, the 1/deviations
    constexpr uint32_t kD = V * sizeof(TD), kX = V * sizeof(TX);
    const uint32_t threads = blockDim.x, stage = threads * bwd_stage_bytes<TD, TX, E>(), x_at = NV * kD * threads, mean_at = x_at + NV * kX * threads;
    auto issue = [&](long long r, uint32_t s) {
        const bool live = r < P.M;
        const long long row = live ? r : 0;
        const TD *dy = static_cast<const TD *>(P.dY) + row * P.lddy + t * V;
        const TX *x = static_cast<const TX *>(P.X) + row * P.ldx + t * V;
        const uint32_t to = smem_u32(bwd_smem) + s * stage;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            // what is not there is copied from the first elements, no byte of it
            const bool there = live && col(j) < C;
            copy_piece<kD>(to + kD * (j * threads + threadIdx.x), there ? dy + j * T * V : static_cast<const TD *>(P.dY), there);
            copy_piece<kX>(to + x_at + kX * (j * threads + threadIdx.x), there ? x + j * T * V : static_cast<const TX *>(P.X), there);
        }
        copy_piece<4>(to + mean_at + 4 * threadIdx.x, P.mean + row, live);
        copy_piece<4>(to + mean_at + 4 * (threads + threadIdx.x), P.rstd + row, live);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    long long r0 = (long long)blockIdx.x * teams;
    uint32_t s_in = kStages - 1, s_out = 0;
    if constexpr (kRing) {
        if (r0 < P.M)
            for (uint32_t k = 0; k < kStages - 1; ++k) issue(r0 + team + k * step, k);
    } else {
        if (r0 < P.M) fetch(r0 + team);
    }
    for (; r0 < P.M; r0 += step) {
        const long long r = r0 + team;
        const bool live = r < P.M;
        two_f32 g[P2], d[P2];                    // dY, then rstd g; X, then X - mean
        float mean, rstd;
        if constexpr (kRing) {
            issue(r + (kStages - 1) * step, s_in);
            if (++s_in == kStages) s_in = 0;
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            const uint8_t *const from = bwd_smem + s_out * stage;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                nd[j].load(reinterpret_cast<const TD *>(from + kD * (j * threads + threadIdx.x)));
                nx[j].load(reinterpret_cast<const TX *>(from + x_at + kX * (j * threads + threadIdx.x)));
            }
            mean = *reinterpret_cast<const float *>(from + mean_at + 4 * threadIdx.x);
            rstd = *reinterpret_cast<const float *>(from + mean_at + 4 * (threads + threadIdx.x));
            if (++s_out == kStages) s_out = 0;
        }
        {
            float fd[E], fx[E];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                nd[j].get(*reinterpret_cast<float(*)[V]>(fd + j * V));
                nx[j].get(*reinterpret_cast<float(*)[V]>(fx + j * V));
            }
#pragma unroll
            for (int i = 0; i < P2; ++i) {
                g[i] = two(fd[2 * i], fd[2 * i + 1]);
                d[i] = two(fx[2 * i], fx[2 * i + 1]);
            }
        }
        if constexpr (!kRing) {
            mean = n_mean;
            rstd = n_rstd;
            if (r0 + step < P.M) fetch(r + step);
        }
        // past the row's end dy and gamma are zero
        const two_f32 minus = two(-mean, -mean), scale = two(rstd, rstd);
        two_f32 s0 = 0, s1 = 0;
#pragma unroll
        for (int i = 0; i < P2; ++i) {
            d[i] = add2(d[i], minus);
            a_b[i] = add2(a_b[i], g[i]);
            g[i] = mul2(g[i], scale);
            a_g[i] = fma2(g[i], d[i], a_g[i]);
            g[i] = mul2(g[i], ga[i]);
            s0 = add2(s0, g[i]);
            s1 = fma2(g[i], d[i], s1);
        }
        if (P.dX == nullptr) continue;
        float s[2] = {sum2(s0), sum2(s1)};
        if constexpr (TT > 0) team_sum<TT>(s, red, turn, barrier);
        else team_sum(s, T, red, turn, barrier);
        if (!live) continue;
        const float c0 = -s[0] * inv, c1 = -s[1] * inv * rstd * rstd;
        const two_f32 k0 = two(c0, c0), k1 = two(c1, c1);
        TO *o = static_cast<TO *>(P.dX) + r * P.lddx;
        float f[E];
#pragma unroll
        for (int i = 0; i < P2; ++i) each(fma2(d[i], k1, add2(g[i], k0)), f[2 * i], f[2 * i + 1]);
        if (P.add)
#pragma unroll
            for (int j = 0; j < NV; ++j) add_vector(*reinterpret_cast<float(*)[V]>(f + j * V), static_cast<const TO *>(P.add) + r * P.lddx, col, j);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (col(j) < C) store(o + col(j), *reinterpret_cast<const float(*)[V]>(f + j * V));
    }
    if constexpr (kRing) {
        // the stages take the sums
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
    }
    float *const cols = reinterpret_cast<float *>(bwd_smem);
    if (P.part == nullptr) return;
    float *out = P.part + (long long)blockIdx.x * 2 * C;
    float g[E], b[E];
#pragma unroll
    for (int i = 0; i < P2; ++i) { each(a_g[i], g[2 * i], g[2 * i + 1]); each(a_b[i], b[2 * i], b[2 * i + 1]); }
    // the teams of a warp by shuffles, then the warps in turn: a fixed order
    for (int o = T; o < 32; o <<= 1)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            g[e] += __shfl_xor_sync(0xffffffffu, g[e], o);
            b[e] += __shfl_xor_sync(0xffffffffu, b[e], o);
        }
    const int span = max(T, 32);
    join_sums<V>(g, b, col, (int)threadIdx.x % span < T, threadIdx.x / span, blockDim.x / span, cols, out);
}

// Rows of more than 8192 elements, through shared memory by bulk copies (see norm_fwd_ring_kernel; up to 8192 it is behind the one above by up to 1.6 times).  The sums over the rows fill the registers, so a row is read
// twice from its stage, for its two sums and for its gradient; the stage is refilled after the next row's sums, when the whole team has
// left it.
template <typename TD, typename TX, typename TO, int V, int E, int TT>
__global__ void __launch_bounds__(kBwdThreads, 1) norm_bwd_ring_kernel(const __grid_constant__ BwdParams P, const __grid_constant__ Ring R)
{
    constexpr int P2 = E / 2, W = V;         // elements worked on at a time
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ unsigned long long full[kMaxTeams][kMaxRing];
    __shared__ __align__(16) float red[2][32][2];
    __shared__ volatile int gave_up;
    unsigned int turn = 0;
    const int T = TT ? TT : P.T, team = threadIdx.x / T, t = threadIdx.x - team * T, C = TT ? TT * E : (int)P.C;
    const int teams = blockDim.x / T, barrier = teams > 1 ? team + 1 : 0;
    const float inv = 1.0f / (float)C;
    const Columns<V, TT> col{T, t, C};
    if (t == 0)
        for (int s = 0; s < R.stages; ++s) mbar_init(&full[team][s], 1);
    if (threadIdx.x == 0) gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    pdl_begin();
    uint8_t *const mine = ring + R.params + (size_t)team * R.stages * R.stage_bytes;
    const long long first = (long long)blockIdx.x * teams + team, step = (long long)gridDim.x * teams;
    auto issue = [&](long long r, int s) {
        if (r >= P.M) return;
        uint8_t *const st = mine + (size_t)s * R.stage_bytes;
        mbar_expect_tx(&full[team][s], C * (uint32_t)(sizeof(TD) + sizeof(TX)));
        bulk_load(st, static_cast<const TD *>(P.dY) + r * P.lddy, C * (uint32_t)sizeof(TD), &full[team][s]);
        bulk_load(st + R.second, static_cast<const TX *>(P.X) + r * P.ldx, C * (uint32_t)sizeof(TX), &full[team][s]);
    };
    if (t == 0)
        for (int s = 0; s < R.stages; ++s) issue(first + s * step, s);
    const bool in_ring = TT ? TT * E * sizeof(float) <= kBwdRingBytes / 2 : R.params > 0;
    float *const gammas = in_ring ? reinterpret_cast<float *>(ring) : nullptr;
    if (in_ring) {
        for (int c = threadIdx.x; c < C; c += blockDim.x) gammas[param_at<V>(c, C)] = P.gamma ? P.gamma[c] : 1.0f;
        __syncthreads();
    }
    two_f32 a_g[P2], a_b[P2];
#pragma unroll
    for (int i = 0; i < P2; ++i) a_g[i] = a_b[i] = 0;
    int s = 0;
    uint32_t ph = 0;
    float n_mean = first < P.M ? P.mean[first] : 0.0f, n_rstd = first < P.M ? P.rstd[first] : 0.0f;
    for (long long r = first; r < P.M; r += step) {
        const float mean = n_mean, rstd = n_rstd;
        if (r + step < P.M) { n_mean = P.mean[r + step]; n_rstd = P.rstd[r + step]; }
        const bool ok = mbar_wait(&full[team][s], ph, &gave_up, nullptr, 0);
        const uint8_t *const st = mine + (size_t)s * R.stage_bytes;
        const TX *const x = reinterpret_cast<const TX *>(st + R.second);
        const TD *const dy = reinterpret_cast<const TD *>(st);
        const two_f32 minus = two(-mean, -mean), scale = two(rstd, rstd);
        // W elements from e on: d = x - mean, dy, gamma (past the row's end dy and gamma are zero)
        auto load = [&](int e, two_f32 (&d)[W / 2], two_f32 (&g)[W / 2], two_f32 (&ga)[W / 2]) {
            float fx[W], fd[W], fg[W];
            const int j = e / V;
            read_vector(x, col, j, fx);
            read_vector(dy, col, j, fd);
            if (col.whole(j) || col(j) < C) {
                read_param<V>(gammas, P.gamma, col(j), C, 1.0f, fg);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) fg[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
                d[i] = add2(two(fx[2 * i], fx[2 * i + 1]), minus);
                g[i] = two(fd[2 * i], fd[2 * i + 1]);
                ga[i] = two(fg[2 * i], fg[2 * i + 1]);
            }
        };
        two_f32 s0 = 0, s1 = 0;
#pragma unroll
        for (int e = 0; e < E; e += W) {
            two_f32 d[W / 2], g[W / 2], ga[W / 2];
            load(e, d, g, ga);
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
                a_b[e / 2 + i] = add2(a_b[e / 2 + i], g[i]);
                g[i] = mul2(g[i], scale);
                a_g[e / 2 + i] = fma2(g[i], d[i], a_g[e / 2 + i]);
                g[i] = mul2(g[i], ga[i]);
                s0 = add2(s0, g[i]);
                s1 = fma2(g[i], d[i], s1);
            }
        }
        float sums[2] = {sum2(s0), ok ? sum2(s1) : __uint_as_float(0x7FC00000u)};
        if constexpr (TT > 0) team_sum<TT>(sums, red, turn, barrier);
        else team_sum(sums, T, red, turn, barrier);
        // the whole team has left the row before this one: its stage is free
        if (T == 32) __syncwarp();
        if (t == 0 && r != first) issue(r + (R.stages - 1) * step, s == 0 ? R.stages - 1 : s - 1);
        if (P.dX) {
            const float c0 = -sums[0] * inv, c1 = -sums[1] * inv * rstd * rstd;
            const two_f32 k0 = two(c0, c0), k1 = two(c1, c1);
            TO *o = static_cast<TO *>(P.dX) + r * P.lddx;
            const TO *const add = P.add ? static_cast<const TO *>(P.add) + r * P.lddx : nullptr;
#pragma unroll
            for (int e = 0; e < E; e += W) {
                two_f32 d[W / 2], g[W / 2], ga[W / 2];
                load(e, d, g, ga);
                float f[W];
#pragma unroll
                for (int i = 0; i < W / 2; ++i) each(fma2(d[i], k1, fma2(g[i], mul2(ga[i], scale), k0)), f[2 * i], f[2 * i + 1]);
                const int j = e / V;
                if (add) add_vector(f, add, col, j);
                if (col.whole(j) || col(j) < C) store(o + col(j), f);
            }
        }
        if (++s == R.stages) { s = 0; ph ^= 1u; }
    }
    if (P.part == nullptr) return;
    __syncthreads();                         // no copy is on its way: the ring takes the sums, the teams in turn
    float *const cols = reinterpret_cast<float *>(ring), *const out = P.part + (long long)blockIdx.x * 2 * C;
    float g[E], b[E];
#pragma unroll
    for (int i = 0; i < P2; ++i) { each(a_g[i], g[2 * i], g[2 * i + 1]); each(a_b[i], b[2 * i], b[2 * i + 1]); }
    join_sums<V>(g, b, col, true, team, teams, cols, out);
}

// Long rows, first pass: sum(g) / C and sum(g xh) / C of every row.
template <typename TD, typename TX, int V>
__global__ void __launch_bounds__(kBwdThreads) norm_bwd_sums_kernel(const __grid_constant__ BwdParams P)
{
    __shared__ __align__(16) float red[2][32][2];
    unsigned int turn = 0;
    const float inv = 1.0f / (float)P.C;
    pdl_begin();
    for (long long r = blockIdx.x; r < P.M; r += gridDim.x) {
        const TD *dy = static_cast<const TD *>(P.dY) + r * P.lddy;
        const TX *xr = static_cast<const TX *>(P.X) + r * P.ldx;
        const float mean = P.mean[r], rstd = P.rstd[r];
        float s[2] = {0.0f, 0.0f};
        for (long long col = (long long)threadIdx.x * V; col < P.C; col += kBwdThreads * V) {
            Vec<TD, V> vd;
            Vec<TX, V> vx;
            float d[V], x[V], ga[V];
            vd.load(dy + col);
            vx.load(xr + col);
            vd.get(d);
            vx.get(x);
            load_param(ga, P.gamma, col, 1.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float g = d[i] * ga[i];
                s[0] += g;
                s[1] = fmaf(g, (x[i] - mean) * rstd, s[1]);
            }
        }
        team_sum(s, kBwdThreads, red, turn, 0);
        if (threadIdx.x == 0) {
            P.row_sums[2 * r] = s[0] * inv;
            P.row_sums[2 * r + 1] = s[1] * inv;
        }
    }
}

// Long rows, second pass: a block has a stripe of columns and every parts-th row; no sums across threads are left.
constexpr int kStripeThreads = 256;
template <typename TD, typename TX, typename TO, int V>
__global__ void __launch_bounds__(kStripeThreads) norm_bwd_stripe_kernel(const __grid_constant__ BwdParams P)
{
    const long long col = ((long long)blockIdx.x * kStripeThreads + threadIdx.x) * V;
    const int part = blockIdx.y;
    pdl_begin();
    if (col >= P.C) return;
    float ga[V], a_g[V], a_b[V];
    load_param(ga, P.gamma, col, 1.0f);
#pragma unroll
    for (int i = 0; i < V; ++i) a_g[i] = a_b[i] = 0.0f;
#pragma unroll 4
    for (long long r = part; r < P.M; r += P.parts) {
        Vec<TD, V> vd;
        Vec<TX, V> vx;
        float d[V], x[V];
        vd.load(static_cast<const TD *>(P.dY) + r * P.lddy + col);
        vx.load(static_cast<const TX *>(P.X) + r * P.ldx + col);
        const float mean = P.mean[r], rstd = P.rstd[r], c0 = P.row_sums[2 * r], c1 = P.row_sums[2 * r + 1];
        vd.get(d);
        vx.get(x);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float xh = (x[i] - mean) * rstd;
            a_g[i] = fmaf(d[i], xh, a_g[i]);
            a_b[i] += d[i];
            d[i] = (fmaf(d[i], ga[i], -c0) - xh * c1) * rstd;
        }
        if (P.dX) {
            if (P.add) {
                Vec<TO, V> w;
                float e[V];
                w.load(static_cast<const TO *>(P.add) + r * P.lddx + col);
                w.get(e);
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] += e[i];
            }
            store(static_cast<TO *>(P.dX) + r * P.lddx + col, d);
        }
    }
    if (P.part) {
        float *out = P.part + (long long)part * 2 * P.C + col;
        store(out, a_g);
        store(out + P.C, a_b);
    }
}

// dgamma and dbeta: a column's parts in 32 runs, all of a run's loads at once (with eight runs, one load after the other, the fold of 148
// parts took longer than what it folds), and the runs in order.
constexpr int kPartBlocks = 148, kRuns = 32, kPerRun = (kPartBlocks + kRuns - 1) / kRuns;
// W columns a thread, so that up to 4736 channels, or 9472, are a block an SM, which may start early.
template <int W> __global__ void __launch_bounds__(32 * kRuns) norm_fold_kernel(const float *part, int parts, long long C, float *dgamma, float *dbeta)
{
    __shared__ float s[kRuns][32 * W];
    pdl_begin();
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const long long c = ((long long)blockIdx.x * 32 + lane) * W;
    float w[kPerRun][W], v[W];
#pragma unroll
    for (int k = 0; k < kPerRun; ++k) {
        const int p = run + kRuns * k;
#pragma unroll
        for (int i = 0; i < W; ++i) w[k][i] = 0.0f;
        if (p < parts && c < 2 * C) {
            const float *const from = part + (long long)p * 2 * C + c;
            if constexpr (W == 4) {
                const float4 a = __ldg(reinterpret_cast<const float4 *>(from));
                w[k][0] = a.x; w[k][1] = a.y; w[k][2] = a.z; w[k][3] = a.w;
            } else if constexpr (W == 2) {
                const float2 a = __ldg(reinterpret_cast<const float2 *>(from));
                w[k][0] = a.x; w[k][1] = a.y;
            } else {
                w[k][0] = __ldg(from);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        v[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < kPerRun; ++k) v[i] += w[k][i];
        s[run][lane * W + i] = v[i];
    }
    __syncthreads();
    if (run < W) {
        const long long at = (long long)blockIdx.x * 32 * W + threadIdx.x;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kRuns; ++k) sum += s[k][threadIdx.x];
        float *const out = at < C ? dgamma : dbeta;
        if (at < 2 * C && out) out[at < C ? at : at - C] = sum;
    }
}

bool is_dtype(int d) { return d == TWN_F32 || d == TWN_BF16; }
size_t size_of(int d) { return d == TWN_BF16 ? 2 : 4; }

// A matrix of M rows of C elements, ld apart: TWN_OK or why not.
int check_matrix(const void *p, int dtype, long long ld, long long M, long long C)
{
    TWN_REQUIRE(is_dtype(dtype) && ld >= C, TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(M == 0 || p != nullptr, TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(twn_aligned(p, size_of(dtype)), TWN_ERR_MISALIGNED);
    TWN_REQUIRE(M == 0 || ld <= (1ll << 58) / M, TWN_ERR_TOO_LARGE);
    return TWN_OK;
}
// Rows whose runs of V elements are aligned to their loads (of 16 bytes at most).
bool vector_rows(const void *p, int dtype, long long ld, int V)
{
    const long long unit = std::min<long long>(16, V * (long long)size_of(dtype));
    return twn_aligned(p, (size_t)unit) && ld * (long long)size_of(dtype) % unit == 0;
}

constexpr long long kMaxC = 1ll << 31;       // channels: partial sums and columns stay far inside 64 bits
constexpr long long kRingElements = 1 << 20;  // below, the launch itself is what counts

int team_for(long long C, int E, int least, int most)
{
    int T = least;
    while (T < most && (long long)T * E < C) T *= 2;
    return T;
}

template <typename TX, typename TY, int V, int E, int TT> int launch_fwd(FwdParams &P, int T, cudaStream_t s)
{
    P.T = T;
    const int block = T > 32 ? T : 128, teams = block / T;
    const long long grid = std::min<long long>((P.M + teams - 1) / teams, 148ll * 64);
    TWN_CUDA_OK(twn_launch_small(norm_fwd_kernel<TX, TY, V, E, TT>, (int)grid, block, 0, s, P));
    return TWN_OK;
}
// Threads of a row (whole warps), rows that a block has at once, and their rings behind what holds gamma and beta.
struct RingShape {
    int T, teams;
    Ring ring;
    size_t smem;
};
bool ring_shape(RingShape &r, size_t bytes, long long C, int E, int threads, size_t stage, size_t second, size_t params)
{
    r.T = (int)((C + 32 * E - 1) / (32 * E)) * 32;
    if (r.T > threads) return false;
    r.teams = std::min(threads / r.T, r.T > 32 ? 15 : kMaxTeams);          // a block has fifteen named barriers beside its own
    params = (params + 127) / 128 * 128;
    if (params > bytes / 2) params = 0;
    while (r.teams > 1 && 2 * r.teams * stage > bytes - params) --r.teams;
    const int stages = (int)std::min<size_t>(kMaxRing, (bytes - params) / (r.teams * stage));
    r.ring = {stages, (int)stage, (int)second, (int)params};
    r.smem = params + r.teams * stages * stage;
    return stages >= 2 && r.teams * r.T >= 256 + 32;
}
template <typename Kernel> int allow_ring(Kernel kernel, int device, bool (&done)[64])
{
    if (!done[device]) TWN_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFwdRingBytes));
    done[device] = true;
    return TWN_OK;
}
template <typename TX, typename TY, int V, int E, int TT> int launch_fwd_ring(const FwdParams &P, const RingShape &r, const twn_device_info &dev, cudaStream_t s)
{
    static bool done[64] = {false};
    const int rc = allow_ring(norm_fwd_ring_kernel<TX, TY, V, E, TT>, dev.ordinal, done);
    if (rc != TWN_OK) return rc;
    const int grid = (int)std::min<long long>((P.M + r.teams - 1) / r.teams, dev.sm_count);
    TWN_CUDA_OK(twn_launch_small(norm_fwd_ring_kernel<TX, TY, V, E, TT>, grid, r.T * r.teams, r.smem, s, P, r.ring));
    return TWN_OK;
}
template <typename TX, typename TY, int V, int E> bool fwd_ring(FwdParams &P, const twn_device_info &dev, cudaStream_t s, int &rc)
{
    RingShape r;
    if (!ring_shape(r, kFwdRingBytes, P.C, E, fwd_ring_threads<E>(), P.C * sizeof(TX), 0, 2 * sizeof(float) * P.C)) return false;
    P.T = r.T;
    const int filled = P.C == (long long)r.T * E ? r.T : 0;
    if constexpr (E == 64) {
        rc = filled == 32    ? launch_fwd_ring<TX, TY, V, E, 32>(P, r, dev, s)
             : filled == 64  ? launch_fwd_ring<TX, TY, V, E, 64>(P, r, dev, s)
             : filled == 128 ? launch_fwd_ring<TX, TY, V, E, 128>(P, r, dev, s)
             : filled == 256 ? launch_fwd_ring<TX, TY, V, E, 256>(P, r, dev, s)
             : filled == 512 ? launch_fwd_ring<TX, TY, V, E, 512>(P, r, dev, s)
                             : launch_fwd_ring<TX, TY, V, E, 0>(P, r, dev, s);
    } else {
        rc = filled == 32 ? launch_fwd_ring<TX, TY, V, E, 32>(P, r, dev, s) : launch_fwd_ring<TX, TY, V, E, 0>(P, r, dev, s);
    }
    return true;
}
template <typename TD, typename TX, typename TO, int V, int E, int TT>
int launch_bwd_ring(const BwdParams &P, const RingShape &r, const twn_device_info &dev, cudaStream_t s)
{
    static bool done[64] = {false};
    const int rc = allow_ring(norm_bwd_ring_kernel<TD, TX, TO, V, E, TT>, dev.ordinal, done);
    if (rc != TWN_OK) return rc;
    TWN_CUDA_OK(twn_launch_small(norm_bwd_ring_kernel<TD, TX, TO, V, E, TT>, P.parts, r.T * r.teams, r.smem, s, P, r.ring));
    return TWN_OK;
}
template <typename TD, typename TX, typename TO, int V, int E> bool bwd_ring(BwdParams &P, const twn_device_info &dev, cudaStream_t s, int &rc)
{
    RingShape r;
    const size_t second = P.C * sizeof(TD);
    if (!ring_shape(r, kBwdRingBytes, P.C, E, kBwdThreads, second + P.C * sizeof(TX), second, sizeof(float) * P.C)) return false;
    P.T = r.T;
    P.parts = (int)std::min<long long>((P.M + r.teams - 1) / r.teams, std::min(dev.sm_count, kPartBlocks));
    // at most 512 threads of 32 columns: 128 KB
    r.smem = std::max<size_t>(r.smem, r.teams > 1 ? r.teams * 2 * sizeof(float) * P.C : 0);
    const int filled = P.C == (long long)r.T * E ? r.T : 0;
    rc = filled == 512 ? launch_bwd_ring<TD, TX, TO, V, E, 512>(P, r, dev, s) : launch_bwd_ring<TD, TX, TO, V, E, 0>(P, r, dev, s);
    return true;
}

template <typename TX, typename TY, int V> int fwd(FwdParams &P, const twn_device_info &dev, cudaStream_t s)
{
    if constexpr (V > 1) {
        int rc = TWN_OK;
        if (P.C > 256 && P.M * P.C >= kRingElements &&
            (P.C <= 512 ? fwd_ring<TX, TY, V, 16>(P, dev, s, rc)
             : P.C <= 1024 ? fwd_ring<TX, TY, V, 32>(P, dev, s, rc)
                           : fwd_ring<TX, TY, V, 64>(P, dev, s, rc)))
            return rc;
    }
    if (P.C <= 32 * 8) return launch_fwd<TX, TY, V, 8, 0>(P, team_for(P.C, 8, 4, 32), s);
    if constexpr (V > 1) {
        if (P.C <= 512) return launch_fwd<TX, TY, V, 16, 32>(P, 32, s);
        if (P.C <= 1024) return launch_fwd<TX, TY, V, 16, 64>(P, 64, s);
        if (P.C <= 2048) return launch_fwd<TX, TY, V, 16, 128>(P, 128, s);
        if (P.C <= 4096) return launch_fwd<TX, TY, V, 16, 256>(P, 256, s);
        if (P.C <= 8192) return launch_fwd<TX, TY, V, 16, 512>(P, 512, s);
        if (P.C <= 16384) return launch_fwd<TX, TY, V, 32, 512>(P, 512, s);
        if (P.C <= 32768) return launch_fwd<TX, TY, V, 32, 1024>(P, 1024, s);
    } else {
        if (P.C <= 512) return launch_fwd<TX, TY, 1, 16, 32>(P, 32, s);
        if (P.C <= 1024) return launch_fwd<TX, TY, 1, 16, 64>(P, 64, s);
        if (P.C <= 2048) return launch_fwd<TX, TY, 1, 16, 128>(P, 128, s);
        if (P.C <= 4096) return launch_fwd<TX, TY, 1, 16, 256>(P, 256, s);
        if (P.C <= 8192) return launch_fwd<TX, TY, 1, 16, 512>(P, 512, s);
        if (P.C <= 16384) return launch_fwd<TX, TY, 1, 16, 1024>(P, 1024, s);
    }
    const int grid = (int)std::min<long long>(P.M, 148 * 2);
    TWN_CUDA_OK(twn_launch_small(norm_fwd_long_kernel<TX, TY, V>, grid, 1024, 0, s, P));
    return TWN_OK;
}
template <typename TX, typename TY> int fwd_any(FwdParams &P, bool vec, const twn_device_info &dev, cudaStream_t s)
{
    constexpr int V = sizeof(TX) == 2 ? 8 : 4;
    return vec ? fwd<TX, TY, V>(P, dev, s) : fwd<TX, TY, 1>(P, dev, s);
}

template <typename TD, typename TX, typename TO, int V, int E, int TT>
int launch_bwd_rows(BwdParams &P, int threads, size_t smem, const twn_device_info &dev, cudaStream_t s)
{
    static bool done[64] = {false};
    const int rc = allow_ring(norm_bwd_kernel<TD, TX, TO, V, E, TT>, dev.ordinal, done);
    if (rc != TWN_OK) return rc;
    TWN_CUDA_OK(twn_launch_small(norm_bwd_kernel<TD, TX, TO, V, E, TT>, P.parts, threads, smem, s, P));
    return TWN_OK;
}
template <typename TD, typename TX, typename TO, int V, int E> int bwd_rows(BwdParams &P, const twn_device_info &dev, cudaStream_t s)
{
    P.T = team_for(P.C, E, 4, kBwdThreads);
    // few rows: blocks of fewer teams, so that there are more of them
    int threads = kBwdThreads;
    while (threads > std::max(P.T, 128) && (P.M * P.T + threads - 1) / threads < dev.sm_count) threads /= 2;
    const int teams = threads / P.T;
    P.parts = (int)std::max<long long>(1, std::min<long long>((P.M + teams - 1) / teams, std::min(dev.sm_count, kPartBlocks)));
    const int parties = threads / std::max(P.T, 32);
    const size_t sums = parties > 1 && P.part ? parties * 2 * sizeof(float) * P.C : 0;
    const size_t smem = V > 1 ? std::max<size_t>(sums, (size_t)bwd_stages<TD, TX>() * threads * bwd_stage_bytes<TD, TX, E>()) : sums;
    switch (P.T) {
        case 4: return launch_bwd_rows<TD, TX, TO, V, E, V == 1 ? 0 : 4>(P, threads, smem, dev, s);
        case 8: return launch_bwd_rows<TD, TX, TO, V, E, V == 1 ? 0 : 8>(P, threads, smem, dev, s);
        case 16: return launch_bwd_rows<TD, TX, TO, V, E, V == 1 ? 0 : 16>(P, threads, smem, dev, s);
        case 32: return launch_bwd_rows<TD, TX, TO, V, E, 32>(P, threads, smem, dev, s);
        case 64: return launch_bwd_rows<TD, TX, TO, V, E, 64>(P, threads, smem, dev, s);
        case 128: return launch_bwd_rows<TD, TX, TO, V, E, 128>(P, threads, smem, dev, s);
        case 256: return launch_bwd_rows<TD, TX, TO, V, E, 256>(P, threads, smem, dev, s);
        default: return launch_bwd_rows<TD, TX, TO, V, E, 512>(P, threads, smem, dev, s);
    }
}
template <typename TD, typename TX, typename TO, int V> int bwd(BwdParams &P, float *dgamma, float *dbeta, const twn_device_info &dev, cudaStream_t s)
{
    constexpr int E = V > 1 ? 16 : 8;
    int rc = TWN_OK;
    bool served = false;
    if constexpr (V > 1) served = P.bulk && P.C > kBwdThreads * E && P.M * P.C >= kRingElements && bwd_ring<TD, TX, TO, V, 32>(P, dev, s, rc);
    if (served) {
        if (rc != TWN_OK) return rc;
    } else if (V == 1 && P.C <= kBwdThreads * 16 && (P.C > kBwdThreads * E || P.M * P.C >= 1 << 23)) {
        // single elements of large tensors: 60000 x 1001 144 us with eight a thread, 90 with sixteen (2999 x 1001 10.6 and 13.6)
        rc = bwd_rows<TD, TX, TO, V, V == 1 ? 16 : E>(P, dev, s);
        if (rc != TWN_OK) return rc;
    } else if (P.C <= kBwdThreads * E) {
        rc = bwd_rows<TD, TX, TO, V, E>(P, dev, s);
        if (rc != TWN_OK) return rc;
    } else {
        if (P.dX && P.M > 0)
            TWN_CUDA_OK(twn_launch_small(norm_bwd_sums_kernel<TD, TX, V>, (int)std::min<long long>(P.M, 148 * 4), kBwdThreads, 0, s, P));
        const long long stripes = (P.C + kStripeThreads * V - 1) / (kStripeThreads * V);
        P.parts = (int)std::max<long long>(1, std::min<long long>(std::min<long long>(P.M, kPartBlocks), 148 * 8 / stripes));
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)stripes, (unsigned)P.parts);
        cfg.blockDim = dim3(kStripeThreads);
        cfg.stream = s;
        TWN_CUDA_OK(cudaLaunchKernelEx(&cfg, norm_bwd_stripe_kernel<TD, TX, TO, V>, P));
    }
    if (P.part == nullptr) return TWN_OK;
    auto fold = [&](auto kernel, int W) {
        return twn_launch_small(kernel, (int)((2 * P.C + 32 * W - 1) / (32 * W)), 32 * kRuns, 0, s, P.part, P.parts, P.C, dgamma, dbeta);
    };
    const long long narrow = 16 * kPdlBlocks;            // channels whose columns, one a thread, are that many blocks
    TWN_CUDA_OK(P.C <= narrow || P.C % 2 ? fold(norm_fold_kernel<1>, 1) : P.C <= 2 * narrow || P.C % 4 ? fold(norm_fold_kernel<2>, 2) : fold(norm_fold_kernel<4>, 4));
    return TWN_OK;
}
template <typename TD, typename TX, typename TO>
int bwd_any(BwdParams &P, bool vec, float *dgamma, float *dbeta, const twn_device_info &dev, cudaStream_t s)
{
    constexpr int V = sizeof(TD) == 4 || sizeof(TX) == 4 ? 4 : 8;
    return vec ? bwd<TD, TX, TO, V>(P, dgamma, dbeta, dev, s) : bwd<TD, TX, TO, 1>(P, dgamma, dbeta, dev, s);
}

size_t align256(size_t v) { return (v + 255) / 256 * 256; }
size_t part_bytes(int64_t C) { return align256(size_t(kPartBlocks) * 2 * sizeof(float) * (size_t)C); }

}  // namespace

extern "C" int twn_layer_norm_fwd(const void *X, int32_t x_dtype, int64_t ldx, int64_t M, int64_t C, const float *gamma,
                                  const float *beta, double eps, void *Y, int32_t y_dtype, int64_t ldy, float *mean, float *rstd,
                                  twn_stream_t stream)
{
    TWN_REQUIRE(M >= 0 && C >= 1 && C <= kMaxC && std::isfinite(eps) && eps >= 0.0, TWN_ERR_INVALID_ARG);
    int rc = check_matrix(X, x_dtype, ldx, M, C);
    if (rc == TWN_OK) rc = check_matrix(Y, y_dtype, ldy, M, C);
    if (rc != TWN_OK) return rc;
    for (const void *p : {(const void *)gamma, (const void *)beta, (const void *)mean, (const void *)rstd})
        TWN_REQUIRE(twn_aligned(p, 4), TWN_ERR_MISALIGNED);
    if (M == 0) return TWN_OK;
    twn_device_info dev;
    rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    FwdParams P = {X, Y, gamma, beta, mean, rstd, ldx, ldy, M, C, (float)eps, 0};
    const int V = x_dtype == TWN_BF16 ? 8 : 4;
    const bool vec = vector_rows(X, x_dtype, ldx, V) && vector_rows(Y, y_dtype, ldy, V) && C % V == 0 && twn_aligned(gamma, 16) &&
                     twn_aligned(beta, 16);
    cudaStream_t s = twn_cu(stream);
    if (x_dtype == TWN_BF16) return y_dtype == TWN_BF16 ? fwd_any<bf16, bf16>(P, vec, dev, s) : fwd_any<bf16, float>(P, vec, dev, s);
    return y_dtype == TWN_BF16 ? fwd_any<float, bf16>(P, vec, dev, s) : fwd_any<float, float>(P, vec, dev, s);
}

extern "C" size_t twn_layer_norm_bwd_workspace_bytes(int64_t M, int64_t C)
{
    if (M < 0 || C < 1 || C > kMaxC || M > (1ll << 58) / C) return 0;
    return part_bytes(C) + align256(2 * sizeof(float) * (size_t)M);
}

extern "C" int twn_layer_norm_bwd(const void *dY, int32_t dy_dtype, int64_t lddy, const void *X, int32_t x_dtype, int64_t ldx,
                                  int64_t M, int64_t C, const float *gamma, const float *mean, const float *rstd, void *dX,
                                  int32_t dx_dtype, int64_t lddx, const void *residual, float *dgamma, float *dbeta,
                                  void *workspace, size_t workspace_bytes, twn_stream_t stream)
{
    TWN_REQUIRE(M >= 0 && C >= 1 && C <= kMaxC, TWN_ERR_INVALID_ARG);
    int rc = check_matrix(dY, dy_dtype, lddy, M, C);
    if (rc == TWN_OK) rc = check_matrix(X, x_dtype, ldx, M, C);
    if (rc == TWN_OK && dX) rc = check_matrix(dX, dx_dtype, lddx, M, C);
    if (rc == TWN_OK && residual) rc = dX ? check_matrix(residual, dx_dtype, lddx, M, C) : TWN_ERR_INVALID_ARG;
    if (rc != TWN_OK) return rc;
    TWN_REQUIRE(M == 0 || (mean != nullptr && rstd != nullptr), TWN_ERR_INVALID_ARG);
    for (const void *p : {(const void *)gamma, (const void *)mean, (const void *)rstd, (const void *)dgamma, (const void *)dbeta})
        TWN_REQUIRE(twn_aligned(p, 4), TWN_ERR_MISALIGNED);
    if (dX == nullptr && dgamma == nullptr && dbeta == nullptr) return TWN_OK;
    TWN_REQUIRE(workspace != nullptr && workspace_bytes >= twn_layer_norm_bwd_workspace_bytes(M, C), TWN_ERR_WORKSPACE);
    TWN_REQUIRE(twn_aligned(workspace, 256), TWN_ERR_MISALIGNED);
    const bool sums = dgamma != nullptr || dbeta != nullptr;
    if (M == 0 && !sums) return TWN_OK;
    twn_device_info dev;
    rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    BwdParams P = {};
    P.dY = dY; P.X = X; P.dX = dX; P.add = residual;
    P.gamma = gamma; P.mean = mean; P.rstd = rstd;
    P.part = sums ? static_cast<float *>(workspace) : nullptr;
    P.row_sums = reinterpret_cast<float *>(static_cast<char *>(workspace) + part_bytes(C));
    P.lddy = lddy; P.ldx = ldx; P.lddx = lddx; P.M = M; P.C = C;
    // vectors of 16 bytes of the wider type, so that a warp's copies are next to each other
    const int V = dy_dtype == TWN_F32 || x_dtype == TWN_F32 ? 4 : 8;
    const bool vec = vector_rows(dY, dy_dtype, lddy, V) && vector_rows(X, x_dtype, ldx, V) && (!dX || vector_rows(dX, dx_dtype, lddx, V)) && (!residual || vector_rows(residual, dx_dtype, lddx, V)) &&
                     C % V == 0 && twn_aligned(gamma, 16);
    P.bulk = C % 8 == 0 && vector_rows(dY, dy_dtype, lddy, 8) && vector_rows(X, x_dtype, ldx, 8);
    cudaStream_t s = twn_cu(stream);
    const int key = (dy_dtype == TWN_BF16) * 4 + (x_dtype == TWN_BF16) * 2 + (dX && dx_dtype == TWN_BF16);
    switch (key) {
        case 0: return bwd_any<float, float, float>(P, vec, dgamma, dbeta, dev, s);
        case 1: return bwd_any<float, float, bf16>(P, vec, dgamma, dbeta, dev, s);
        case 2: return bwd_any<float, bf16, float>(P, vec, dgamma, dbeta, dev, s);
        case 3: return bwd_any<float, bf16, bf16>(P, vec, dgamma, dbeta, dev, s);
        case 4: return bwd_any<bf16, float, float>(P, vec, dgamma, dbeta, dev, s);
        case 5: return bwd_any<bf16, float, bf16>(P, vec, dgamma, dbeta, dev, s);
        case 6: return bwd_any<bf16, bf16, float>(P, vec, dgamma, dbeta, dev, s);
        default: return bwd_any<bf16, bf16, bf16>(P, vec, dgamma, dbeta, dev, s);
    }
}
