// Layer norm over the channels of a row (a token, or a pixel of an NHWC tensor), forward and backward.
//
//   forward   mean = sum x / C,  var = sum (x - mean)^2 / C,  rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd gamma + beta
//   backward  xh = (x - mean) rstd,  g = dy gamma,  dx = rstd (g - sum(g) / C - xh sum(g xh) / C),
//             dgamma = sum over the rows of dy xh,  dbeta = sum over the rows of dy
//
// Both are bound by HBM: a row is read once and stays in registers until its result is written.  A team of T threads (4 to
// 1024, a power of two) has a row, E elements a thread; its sums are shuffle trees, and one barrier where it is more than a
// warp.  The variance is that of the differences from the mean (a second tree), never a difference of two sums: rows far from
// zero keep their digits.  All arithmetic is fp32, rounded once to the type of the output.
#include <algorithm>
#include <cmath>

#include <cuda_bf16.h>

#include "common.cuh"

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

// gamma and beta: fp32, `none` where the caller has none
template <int V> __device__ __forceinline__ void load_param(float (&f)[V], const float *p, long long col, float none)
{
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = none;
    } else {
        Vec<float, V> v;
        v.load(p + col);
        v.get(f);
    }
}

// Sums over a team of T threads, the same bits in all of them.  Every thread of the block calls it.  `red` holds N floats for
// each of 32 warps, twice: a buffer is written again one barrier after all have read it.
template <int N> __device__ __forceinline__ void team_sum(float (&v)[N], int T, float (*red)[32][2], unsigned int &turn)
{
    const int span = min(T, 32);
    for (int o = span >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (T > 32) {
        float(*buf)[2] = red[turn & 1];
        ++turn;
        const int warp = threadIdx.x >> 5, warps = T >> 5;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) buf[warp][i] = v[i];
        __syncthreads();
        const int first = warp & ~(warps - 1), lane = threadIdx.x & 31;
        const bool in = lane < warps;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = in ? buf[first + lane][i] : 0.0f;
        for (int o = warps >> 1; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, v[i], 0);
    }
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

// One row per team, in registers.  C <= T * E.
template <typename TX, typename TY, int V, int E>
__global__ void __launch_bounds__(1024) norm_fwd_kernel(const __grid_constant__ FwdParams P)
{
    constexpr int NV = E / V;
    __shared__ float red[2][32][2];
    unsigned int turn = 0;
    const int T = P.T, t = threadIdx.x & (T - 1);
    const int teams = blockDim.x / T, team = threadIdx.x / T;
    const float inv = 1.0f / (float)P.C;
    pdl_begin();
    for (long long r0 = (long long)blockIdx.x * teams; r0 < P.M; r0 += (long long)gridDim.x * teams) {
        const long long r = r0 + team;
        const bool live = r < P.M;
        const TX *x = static_cast<const TX *>(P.X) + (live ? r : 0) * P.ldx;
        Vec<TX, V> raw[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const long long col = (long long)(j * T + t) * V;
            if (live && col < P.C) raw[j].load(x + col);
            else raw[j].zero();
        }
        float f[NV][V], s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            raw[j].get(f[j]);
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += f[j][i];
        }
        team_sum(s, T, red, turn);
        const float mean = s[0] * inv;
        float q[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const bool in = (long long)(j * T + t) * V < P.C;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f[j][i] -= mean;
                if (in) q[0] = fmaf(f[j][i], f[j][i], q[0]);
            }
        }
        team_sum(q, T, red, turn);
        const float rstd = 1.0f / sqrtf(fmaf(q[0], inv, P.eps));
        if (!live) continue;
        TY *y = static_cast<TY *>(P.Y) + r * P.ldy;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const long long col = (long long)(j * T + t) * V;
            if (col >= P.C) continue;
            float ga[V], be[V];
            load_param(ga, P.gamma, col, 1.0f);
            load_param(be, P.beta, col, 0.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) ga[i] = fmaf(f[j][i] * rstd, ga[i], be[i]);
            store(y + col, ga);
        }
        if (t == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
    }
}

// Rows longer than the registers of a block: the row is read three times, from L2 after the first.
template <typename TX, typename TY, int V>
__global__ void __launch_bounds__(1024) norm_fwd_long_kernel(const __grid_constant__ FwdParams P)
{
    __shared__ float red[2][32][2];
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
        team_sum(s, 1024, red, turn);
        const float mean = s[0] * inv;
        float q[1] = {0.0f};
        for (long long col = (long long)threadIdx.x * V; col < P.C; col += 1024 * V) {
            Vec<TX, V> v;
            v.load(x + col);
            v.get(f);
#pragma unroll
            for (int i = 0; i < V; ++i) q[0] = fmaf(f[i] - mean, f[i] - mean, q[0]);
        }
        team_sum(q, 1024, red, turn);
        const float rstd = 1.0f / sqrtf(fmaf(q[0], inv, P.eps));
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
    const float *gamma, *mean, *rstd;
    float *part;                 // [parts][2][C]: sums of dy xh, sums of dy; NULL where the caller wants neither
    float *row_sums;             // long rows: [M][2]
    long long lddy, ldx, lddx, M, C;
    int T, parts;
};

constexpr int kBwdThreads = 512;

// One row per team, the next row's loads in flight while this one is worked on; sums over the rows of a block stay in the
// registers of the threads that own the columns, and its teams join them in shared memory at the end.  C <= T * E.
template <typename TD, typename TX, typename TO, int V, int E>
__global__ void __launch_bounds__(kBwdThreads, 1) norm_bwd_kernel(const __grid_constant__ BwdParams P)
{
    constexpr int NV = E / V;
    extern __shared__ float cols[];          // [2][C], when a block has several teams (of a warp or more)
    __shared__ float red[2][32][2];
    unsigned int turn = 0;
    const int T = P.T, t = threadIdx.x & (T - 1);
    const int teams = kBwdThreads / T, team = threadIdx.x / T;
    const float inv = 1.0f / (float)P.C;
    const long long step = (long long)gridDim.x * teams;
    pdl_begin();
    float ga[NV][V], a_g[NV][V], a_b[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const long long col = (long long)(j * T + t) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) a_g[j][i] = a_b[j][i] = ga[j][i] = 0.0f;
        if (col < P.C) load_param(ga[j], P.gamma, col, 1.0f);
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
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const long long col = (long long)(j * T + t) * V;
            if (live && col < P.C) { nd[j].load(d + col); nx[j].load(x + col); }
            else { nd[j].zero(); nx[j].zero(); }
        }
    };
    long long r0 = (long long)blockIdx.x * teams;
    if (r0 < P.M) fetch(r0 + team);
    for (; r0 < P.M; r0 += step) {
        const long long r = r0 + team;
        const bool live = r < P.M;
        Vec<TD, V> cd[NV];
        Vec<TX, V> cx[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) { cd[j] = nd[j]; cx[j] = nx[j]; }
        const float mean = n_mean, rstd = n_rstd;
        if (r0 + step < P.M) fetch(r + step);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!live || (long long)(j * T + t) * V >= P.C) continue;
            float d[V], x[V];
            cd[j].get(d);
            cx[j].get(x);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (x[i] - mean) * rstd, g = d[i] * ga[j][i];
                s[0] += g;
                s[1] = fmaf(g, xh, s[1]);
                a_g[j][i] = fmaf(d[i], xh, a_g[j][i]);
                a_b[j][i] += d[i];
            }
        }
        if (P.dX == nullptr) continue;
        team_sum(s, T, red, turn);
        if (!live) continue;
        const float c0 = s[0] * inv, c1 = s[1] * inv;
        TO *o = static_cast<TO *>(P.dX) + r * P.lddx;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const long long col = (long long)(j * T + t) * V;
            if (col >= P.C) continue;
            float d[V], x[V];
            cd[j].get(d);
            cx[j].get(x);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (x[i] - mean) * rstd;
                d[i] = (fmaf(d[i], ga[j][i], -c0) - xh * c1) * rstd;
            }
            store(o + col, d);
        }
    }
    if (P.part == nullptr) return;
    float *out = P.part + (long long)blockIdx.x * 2 * P.C;
    // the teams of a warp by shuffles, then the warps in turn: a fixed order
    for (int o = T; o < 32; o <<= 1)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                a_g[j][i] += __shfl_xor_sync(0xffffffffu, a_g[j][i], o);
                a_b[j][i] += __shfl_xor_sync(0xffffffffu, a_b[j][i], o);
            }
    const int span = max(T, 32), turns = kBwdThreads / span;
    for (int k = 0; k < turns; ++k) {
        if ((int)threadIdx.x / span == k && (int)threadIdx.x % span < T)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const long long col = (long long)(j * T + t) * V;
                if (col >= P.C) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float g = a_g[j][i], b = a_b[j][i];
                    if (k > 0) { g += cols[col + i]; b += cols[P.C + col + i]; }
                    float *to = k == turns - 1 ? out : cols;
                    to[col + i] = g;
                    to[P.C + col + i] = b;
                }
            }
        if (turns > 1) __syncthreads();
    }
}

// Long rows, first pass: sum(g) / C and sum(g xh) / C of every row.
template <typename TD, typename TX, int V>
__global__ void __launch_bounds__(kBwdThreads) norm_bwd_sums_kernel(const __grid_constant__ BwdParams P)
{
    __shared__ float red[2][32][2];
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
        team_sum(s, kBwdThreads, red, turn);
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
        if (P.dX) store(static_cast<TO *>(P.dX) + r * P.lddx + col, d);
    }
    if (P.part) {
        float *out = P.part + (long long)part * 2 * P.C + col;
        store(out, a_g);
        store(out + P.C, a_b);
    }
}

// dgamma and dbeta: the parts of each column in a fixed order, eight runs of them at a time.
__global__ void __launch_bounds__(256) norm_fold_kernel(const float *part, int parts, long long C, float *dgamma, float *dbeta)
{
    __shared__ float s[8][33];
    pdl_begin();
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (c < 2 * C)
        for (int p = run; p < parts; p += 8) v += part[(long long)p * 2 * C + c];
    s[run][lane] = v;
    __syncthreads();
    if (run == 0 && c < 2 * C) {
        v = ((s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane])) + ((s[4][lane] + s[5][lane]) + (s[6][lane] + s[7][lane]));
        float *out = c < C ? dgamma : dbeta;
        if (out) out[c < C ? c : c - C] = v;
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
bool vector_rows(const void *p, int dtype, long long ld) { return twn_aligned(p, 16) && ld * (long long)size_of(dtype) % 16 == 0; }

constexpr long long kMaxC = 1ll << 31;       // channels: partial sums and columns stay far inside 64 bits
constexpr int kPartBlocks = 148;

int team_for(long long C, int E, int least, int most)
{
    int T = least;
    while (T < most && (long long)T * E < C) T *= 2;
    return T;
}

template <typename TX, typename TY, int V, int E> int launch_fwd(FwdParams &P, int T, cudaStream_t s)
{
    P.T = T;
    const int block = std::max(T, 128), teams = block / T;
    const long long grid = std::min<long long>((P.M + teams - 1) / teams, 148ll * 64);
    TWN_CUDA_OK(twn_launch_small(norm_fwd_kernel<TX, TY, V, E>, (int)grid, block, 0, s, P));
    return TWN_OK;
}
template <typename TX, typename TY, int V> int fwd(FwdParams &P, cudaStream_t s)
{
    if (P.C <= 32 * 8) return launch_fwd<TX, TY, V, 8>(P, team_for(P.C, 8, 4, 32), s);
    if (P.C <= (V == 1 ? 16 : 8) * 1024) return launch_fwd<TX, TY, V, 16>(P, team_for(P.C, 16, 32, 1024), s);
    if constexpr (V > 1) {                   // 32 elements of one load each do not fit the registers of 1024 threads
        if (P.C <= 32 * 1024) return launch_fwd<TX, TY, V, 32>(P, team_for(P.C, 32, 512, 1024), s);
    }
    const int grid = (int)std::min<long long>(P.M, 148 * 2);
    TWN_CUDA_OK(twn_launch_small(norm_fwd_long_kernel<TX, TY, V>, grid, 1024, 0, s, P));
    return TWN_OK;
}
template <typename TX, typename TY> int fwd_any(FwdParams &P, bool vec, cudaStream_t s)
{
    constexpr int V = sizeof(TX) == 2 ? 8 : 4;
    return vec ? fwd<TX, TY, V>(P, s) : fwd<TX, TY, 1>(P, s);
}

template <typename TD, typename TX, typename TO, int V> int bwd(BwdParams &P, float *dgamma, float *dbeta, int sms, cudaStream_t s)
{
    constexpr int E = V == 8 && sizeof(TD) == 2 && sizeof(TX) == 2 ? 16 : 8;
    if (P.C <= kBwdThreads * E) {
        P.T = team_for(P.C, E, 4, kBwdThreads);
        const int teams = kBwdThreads / P.T;
        P.parts = (int)std::max<long long>(1, std::min<long long>((P.M + teams - 1) / teams, std::min(sms, kPartBlocks)));
        const size_t smem = teams > 1 && P.part ? 2 * sizeof(float) * P.C : 0;
        TWN_CUDA_OK(twn_launch_small(norm_bwd_kernel<TD, TX, TO, V, E>, P.parts, kBwdThreads, smem, s, P));
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
    if (P.part)
        TWN_CUDA_OK(twn_launch_small(norm_fold_kernel, (int)((2 * P.C + 31) / 32), 256, 0, s, P.part, P.parts, P.C, dgamma, dbeta));
    return TWN_OK;
}
template <typename TD, typename TX, typename TO>
int bwd_any(BwdParams &P, bool vec, float *dgamma, float *dbeta, int sms, cudaStream_t s)
{
    constexpr int V = sizeof(TD) == 4 && sizeof(TX) == 4 ? 4 : 8;
    return vec ? bwd<TD, TX, TO, V>(P, dgamma, dbeta, sms, s) : bwd<TD, TX, TO, 1>(P, dgamma, dbeta, sms, s);
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
    const bool vec = vector_rows(X, x_dtype, ldx) && vector_rows(Y, y_dtype, ldy) && C % 8 == 0 && twn_aligned(gamma, 16) &&
                     twn_aligned(beta, 16);
    cudaStream_t s = twn_cu(stream);
    if (x_dtype == TWN_BF16) return y_dtype == TWN_BF16 ? fwd_any<bf16, bf16>(P, vec, s) : fwd_any<bf16, float>(P, vec, s);
    return y_dtype == TWN_BF16 ? fwd_any<float, bf16>(P, vec, s) : fwd_any<float, float>(P, vec, s);
}

extern "C" size_t twn_layer_norm_bwd_workspace_bytes(int64_t M, int64_t C)
{
    if (M < 0 || C < 1 || C > kMaxC || M > (1ll << 58) / C) return 0;
    return part_bytes(C) + align256(2 * sizeof(float) * (size_t)M);
}

extern "C" int twn_layer_norm_bwd(const void *dY, int32_t dy_dtype, int64_t lddy, const void *X, int32_t x_dtype, int64_t ldx,
                                  int64_t M, int64_t C, const float *gamma, const float *mean, const float *rstd, void *dX,
                                  int32_t dx_dtype, int64_t lddx, float *dgamma, float *dbeta, void *workspace,
                                  size_t workspace_bytes, twn_stream_t stream)
{
    TWN_REQUIRE(M >= 0 && C >= 1 && C <= kMaxC, TWN_ERR_INVALID_ARG);
    int rc = check_matrix(dY, dy_dtype, lddy, M, C);
    if (rc == TWN_OK) rc = check_matrix(X, x_dtype, ldx, M, C);
    if (rc == TWN_OK && dX) rc = check_matrix(dX, dx_dtype, lddx, M, C);
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
    P.dY = dY; P.X = X; P.dX = dX;
    P.gamma = gamma; P.mean = mean; P.rstd = rstd;
    P.part = sums ? static_cast<float *>(workspace) : nullptr;
    P.row_sums = reinterpret_cast<float *>(static_cast<char *>(workspace) + part_bytes(C));
    P.lddy = lddy; P.ldx = ldx; P.lddx = lddx; P.M = M; P.C = C;
    const bool vec = vector_rows(dY, dy_dtype, lddy) && vector_rows(X, x_dtype, ldx) && (!dX || vector_rows(dX, dx_dtype, lddx)) &&
                     C % 8 == 0 && twn_aligned(gamma, 16);
    cudaStream_t s = twn_cu(stream);
    const int key = (dy_dtype == TWN_BF16) * 4 + (x_dtype == TWN_BF16) * 2 + (dX && dx_dtype == TWN_BF16);
    switch (key) {
        case 0: return bwd_any<float, float, float>(P, vec, dgamma, dbeta, dev.sm_count, s);
        case 1: return bwd_any<float, float, bf16>(P, vec, dgamma, dbeta, dev.sm_count, s);
        case 2: return bwd_any<float, bf16, float>(P, vec, dgamma, dbeta, dev.sm_count, s);
        case 3: return bwd_any<float, bf16, bf16>(P, vec, dgamma, dbeta, dev.sm_count, s);
        case 4: return bwd_any<bf16, float, float>(P, vec, dgamma, dbeta, dev.sm_count, s);
        case 5: return bwd_any<bf16, float, bf16>(P, vec, dgamma, dbeta, dev.sm_count, s);
        case 6: return bwd_any<bf16, bf16, float>(P, vec, dgamma, dbeta, dev.sm_count, s);
        default: return bwd_any<bf16, bf16, bf16>(P, vec, dgamma, dbeta, dev.sm_count, s);
    }
}
