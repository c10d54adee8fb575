// Layer norm over the channels of a row (a token, or a pixel of an NHWC tensor), forward and backward.
//
//   forward   mean = sum x / C,  var = sum (x - mean)^2 / C,  rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd gamma + beta
//   backward  xh = (x - mean) rstd,  g = dy gamma,  dx = rstd (g - sum(g) / C - xh sum(g xh) / C),
//             dgamma = sum over the rows of dy xh,  dbeta = sum over the rows of dy
//   computed with d = x - mean and h = rstd g, so that xh is never formed:  dx = h - sum(h) / C - d rstd^2 sum(h d) / C
//
// Both are bound by HBM.  A team of T threads has a row, E elements a thread; its sums are shuffle trees, and one barrier where it is
// more than a warp.  The variance is that of the differences from the mean (a second tree), never a difference of two sums: rows far from
// zero keep their digits.  All arithmetic is fp32, rounded once to the type of the output.
//
//   forward    registers (T a power of two from 4 to 1024): the row is read once and stays there until its result is written; small
//              tensors, single elements, rows of 8193 to 32768.  Large tensors of aligned rows of 257 to 32768 that a ring's two stages
//              hold: bulk copies into shared memory, read once from there (T any number of warps).  Longer rows are read three times, from L2 after the first.
//   backward   rows of up to 8192 (T a power of two from 4 to 512): read once, into shared memory by the threads' own copies, or into registers
//              where elements are single.  Aligned rows of 8193 to 16384: bulk copies into a ring, read twice from there (T any number
//              of warps).  Other rows in two launches that read dY and X each: the rows' sums, then stripes of columns (which do form xh).
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>

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

// ---- rows through shared memory ---------------------------------------------------------------------------------------------
// Large tensors of aligned rows.  With 16 elements a thread, all of them in registers, most instructions are the fixed part of a row: two
// sums, the barriers, the root, the addresses; with more, few rows fit the registers, and too little is on its way.  Here rows come by bulk copies into a ring in shared memory, up to 192 KB an SM on their way, for threads
// of up to 64 elements.
constexpr int kMaxRing = 8, kMaxTeams = 32;
// Of the 227 KB that a block may have; 2.6 KB are barriers and sums.  Forward with 200 KB, two stages at 16384 x 4096 instead of three, took 48.0 us for 46.6;
// backward with 224 KB, three instead of two, 85.7 for 82.2.
constexpr size_t kFwdRingBytes = 224 * 1024, kBwdRingBytes = 200 * 1024;

// Waits for rows.  After one that ran out, in any thread, none counts as over: what the thread adds to is no number from there on (the results of its rows,
// and the sums over the rows), nothing more is copied, and before the block ends the copies on their way have had far more than they need.
// (The flag is read where a row's elements are, so that nothing waits for it: 16384 x 2304 forward took 51.3 us for 49.1 with a flag of each thread before the wait.)
__device__ __forceinline__ bool row_is_there(void *bar, uint32_t phase, volatile int *gave_up, unsigned long long limit_ns = kWaitLimitNs)
{
    const bool over = mbar_wait(bar, phase, gave_up, nullptr, 0, limit_ns);
    return over & (*gave_up == 0);
}
template <int N> __device__ __forceinline__ void drop_sums(two_f32 (&a)[N], two_f32 (&b)[N])
{
    const float nan = __uint_as_float(0x7FC00000u);
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = b[i] = two(nan, nan);
}
__device__ __forceinline__ void leave_rows(volatile int *gave_up)
{
    if (*gave_up)
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
}

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
// Bytes that a call reads or writes: `rows` runs of `width`, `pitch` apart.
struct Place {
    long long begin, pitch, width, rows;
    long long end() const { return begin + (rows - 1) * pitch + width; }
};
Place place_of(const void *p, int dtype, long long ld, long long M, long long C)
{
    const long long size = (long long)size_of(dtype), at = (long long)reinterpret_cast<uintptr_t>(p);
    if (ld == C || M == 1) return {at, M * C * size, M * C * size, 1};
    return {at, ld * size, C * size, M};
}
Place place_of(const void *p, long long bytes) { return {(long long)reinterpret_cast<uintptr_t>(p), bytes, bytes, 1}; }
// Whether two of them share a byte.  Of a's rows the first 64 that reach b are looked at: with one pitch, or where b is one run, two of them
// tell; rows of two pitches that meet only further down are the caller's to avoid.
bool meet(const Place &a, const Place &b)
{
    if (a.begin >= b.end() || b.begin >= a.end()) return false;
    const long long first = std::max(0ll, (b.begin - a.begin - a.width + a.pitch) / a.pitch);
    for (long long i = first; i < std::min(first + 64, a.rows); ++i) {
        const long long lo = a.begin + i * a.pitch, hi = lo + a.width;
        // the first row of b that ends behind lo
        const long long j = lo < b.begin + b.width ? 0 : (lo - b.begin - b.width) / b.pitch + 1;
        if (j < b.rows && b.begin + j * b.pitch < hi) return true;
    }
    return false;
}
// What a call writes lies apart from all else that it reads and writes, but for a matrix of the same place, type and pitch.
struct Places {
    struct One {
        Place at;
        int dtype;               // -1: not a matrix
        bool written;
    } all[12];
    int n = 0;
    void matrix(const void *p, int dtype, long long ld, long long M, long long C, bool written)
    {
        if (p) all[n++] = {place_of(p, dtype, ld, M, C), dtype, written};
    }
    void vector(const void *p, long long bytes, bool written)
    {
        if (p) all[n++] = {place_of(p, bytes), -1, written};
    }
    bool apart() const
    {
        for (int i = 0; i < n; ++i)
            for (int j = i + 1; j < n; ++j) {
                const One &a = all[i], &b = all[j];
                if (!a.written && !b.written) continue;
                const bool same = a.dtype >= 0 && a.dtype == b.dtype && a.at.begin == b.at.begin && a.at.pitch == b.at.pitch && a.at.width == b.at.width;
                if (!same && meet(a.at, b.at)) return false;
            }
        return true;
    }
};
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

}  // namespace
