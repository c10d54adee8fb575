// AdamW steps of many tensors in one launch, with the moments in 32 or in 8 bits, and the norm of all gradients that clips them.
//
//   g = scale dW;  m = b1 m + (1 - b1) g;  v = b2 v + ((1 - b2) g) g
//   W = (1 - lr wd) W - (lr / c1) (m / (sqrt(v) / sqrt(c2) + eps)),  c = 1 - b^steps
//
// Every operation is a separately rounded fp32 operation in this order, lr / c1, 1 / sqrt(c2) and 1 - lr wd are rounded from
// fp64: the result is defined to the bit, as the SGD update's is.  The count of steps lives on the device, so that a captured step counts.
//
// Bound by HBM: 28 bytes a weight with fp32 moments and gradients, 16.03 with moments of 8 bits (two bytes less each with bf16 gradients).
//
// Moments of 8 bits.  128 consecutive weights (a warp's four each) share an exponent byte E for each moment.  A code is a
// float of few bits: m a sign, 4 bits of exponent and 3 of fraction, v 5 and 3, the largest exponent standing for 2^(E-127), the smallest one for
// subnormals.  With x scaled by 2^(127-E) and 2^(15-127) (2^(31-127) for v) the exponent field of the fp32 number is that of the code,
// subnormals included, and the code is its upper bits: no conversion is needed in either direction.  E is the exponent of the block's largest value, one
// more where rounding up would carry into the next, so no code ever overflows.
// Roundings are stochastic: v moves by a thousandth of itself a step, a code by an eighth, and to nearest it would never move.  What is
// added below the code are 16 bits of a hash of the weight's index in its tensor, the seed and the count of steps (the same for all tensors, which so do not depend on each other).  A v that is not zero keeps a code that is not
// zero: m / (0 + eps) would be no step but a jump.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include <cuda_bf16.h>

#include "common.cuh"

namespace {

constexpr int kMaxTensors = 256;         // of a call; their items are a launch's parameters
constexpr int kBlock8 = 128;             // weights that share an exponent
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kChunk = 2048;             // weights of a part of a tensor's sums
constexpr int kRow = 4 * kThreads;       // weights that a block has in one instruction of each thread

struct Item {
    float *W;
    const void *dW;
    void *m, *v;
    uint8_t *m_exp, *v_exp;
    long long n;
    double wd;
    twn_stats_t *stats;
    unsigned int first_chunk, first_part;
    int g_bf16;
};
template <int N> struct Launch {
    int count, advance;
    unsigned int chunks;
    float b1, ob1, b2, ob2, eps;
    double lr, one_minus_b1, one_minus_b2, factor;
    unsigned long long seed;
    twn_adamw_step_t *step;
    const float *grad_scale, *lr_scale;
    double *parts;
    Item item[N];
};

// What all weights of a launch share.
struct Step {
    float scale, a, rs2;
    double lr;
    uint32_t key;
};

// A hash of 32 bits: two rounds of a shift, an exclusive or and a product, which flips every bit of its result with nearly even odds.  Shifts and factors are those that Chris Wellons
// found by search and published for anyone's use (2018).
__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}

// 1 - beta^(steps + 1) from 1 - beta^steps: no cancellation, and zero is where it begins.
__device__ __forceinline__ double next_c(double c, double one_minus_beta) { return fma(1.0 - c, one_minus_beta, c); }

template <int N> __device__ __forceinline__ void begin_step(const Launch<N> &P, Step &s)
{
    if (threadIdx.x == 0) {
        const twn_adamw_step_t st = *P.step;
        const double c1 = next_c(st.c1, P.one_minus_b1), c2 = next_c(st.c2, P.one_minus_b2);
        const double lr = P.lr_scale ? P.lr * (double)*P.lr_scale : P.lr;
        s.scale = P.grad_scale ? *P.grad_scale : 1.0f;
        s.lr = lr;
        s.a = (float)(lr / c1);
        s.rs2 = (float)(1.0 / sqrt(c2));
        s.key = mix((uint32_t)P.seed ^ mix((uint32_t)(P.seed >> 32) ^ mix((uint32_t)(st.steps + 1))));
    }
    __syncthreads();
}
// The last block to come here counts the step: by then all have read it.
template <int N> __device__ __forceinline__ void end_step(const Launch<N> &P)
{
    if (!P.advance || threadIdx.x != 0) return;
    unsigned int old;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(old) : "l"(&P.step->arrived) : "memory");
    if (old != gridDim.x - 1) return;
    P.step->c1 = next_c(P.step->c1, P.one_minus_b1);
    P.step->c2 = next_c(P.step->c2, P.one_minus_b2);
    P.step->steps += 1;
    P.step->arrived = 0;
}

template <int N> __device__ __forceinline__ int item_of(const Launch<N> &P, unsigned int chunk)
{
    int lo = 0;
    if (N > 1)
        for (int hi = P.count; hi - lo > 1;) {
            const int mid = (lo + hi) >> 1;
            if (chunk >= P.item[mid].first_chunk) lo = mid;
            else hi = mid;
        }
    return lo;
}

__device__ __forceinline__ void moments(float g, float &m, float &v, float b1, float ob1, float b2, float ob2)
{
    m = __fadd_rn(__fmul_rn(m, b1), __fmul_rn(g, ob1));
    v = __fadd_rn(__fmul_rn(v, b2), __fmul_rn(__fmul_rn(g, ob2), g));
}
__device__ __forceinline__ float updated(float w, float m, float v, float keep, float a, float rs2, float eps)
{
    const float d = __fadd_rn(__fmul_rn(__fsqrt_rn(v), rs2), eps);
    return __fsub_rn(__fmul_rn(w, keep), __fmul_rn(__fdiv_rn(m, d), a));
}

// Four gradients from element i on; zeros from n on.
__device__ __forceinline__ void load_gradient(const Item &it, long long i, bool whole, float (&g)[4])
{
    if (whole) {
        if (it.g_bf16) {
            const uint2 r = __ldg(reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(it.dW) + i));
            g[0] = __uint_as_float(r.x << 16); g[1] = __uint_as_float(r.x & 0xFFFF0000u);
            g[2] = __uint_as_float(r.y << 16); g[3] = __uint_as_float(r.y & 0xFFFF0000u);
        } else {
            const float4 r = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(it.dW) + i));
            g[0] = r.x; g[1] = r.y; g[2] = r.z; g[3] = r.w;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        g[j] = i + j >= it.n ? 0.0f : it.g_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(it.dW)[i + j]) : static_cast<const float *>(it.dW)[i + j];
}
__device__ __forceinline__ void load_four(const float *p, long long i, long long n, bool whole, float (&f)[4])
{
    if (whole) {
        const float4 r = *reinterpret_cast<const float4 *>(p + i);
        f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = i + j < n ? p[i + j] : 0.0f;
}
__device__ __forceinline__ void store_four(float *p, long long i, long long n, bool whole, const float (&f)[4])
{
    if (whole) {
        *reinterpret_cast<float4 *>(p + i) = make_float4(f[0], f[1], f[2], f[3]);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) p[i + j] = f[j];
}

// The tensor that a chunk is of, found anew when it is past the last one's.
template <int N> struct Cursor {
    int t = 0;
    unsigned int end = 0;
    __device__ __forceinline__ bool go(const Launch<N> &P, unsigned int c)
    {
        if (c < end) return false;
        t = item_of(P, c);
        end = t + 1 < P.count ? P.item[t + 1 < N ? t + 1 : 0].first_chunk : P.chunks;
        return true;
    }
};

// Sum of a block's values, in a fixed order; valid in thread 0.
__device__ __forceinline__ double block_sum(double v, double (&warps)[kWarps])
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
    __syncthreads();                     // what was here before has been read
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
#pragma unroll
        for (int i = 0; i < kWarps; ++i) s += warps[i];
    return s;
}

template <bool FULL> __device__ __forceinline__ void add_sizes(const Item &it, long long i, const float (&w)[4], double &sum)
{
    if (it.stats)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += FULL || i + j < it.n ? (double)fabsf(w[j]) : 0.0;
}

// ---- moments in 32 bits -----------------------------------------------------------------------------------------------------
struct In32 {
    float w[4], g[4], m[4], v[4];
};
template <bool FULL> __device__ __forceinline__ In32 load32(const Item &it, long long i)
{
    In32 in;
    const bool whole = FULL || i + 4 <= it.n;
    load_four(it.W, i, it.n, whole, in.w);
    load_gradient(it, i, whole, in.g);
    load_four(static_cast<float *>(it.m), i, it.n, whole, in.m);
    load_four(static_cast<float *>(it.v), i, it.n, whole, in.v);
    return in;
}
template <bool FULL, int N> __device__ __forceinline__ void step32(const Launch<N> &P, const Step &s, const Item &it, float keep, long long i, In32 in, double &sum)
{
    const bool whole = FULL || i + 4 <= it.n;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        moments(__fmul_rn(in.g[j], s.scale), in.m[j], in.v[j], P.b1, P.ob1, P.b2, P.ob2);
        in.w[j] = updated(in.w[j], in.m[j], in.v[j], keep, s.a, s.rs2, P.eps);
    }
    store_four(static_cast<float *>(it.m), i, it.n, whole, in.m);
    store_four(static_cast<float *>(it.v), i, it.n, whole, in.v);
    store_four(it.W, i, it.n, whole, in.w);
    add_sizes<FULL>(it, i, in.w, sum);
}
// A block has every so many-th chunk, of one tensor as long as they last; a thread's next four weights are on their way while it works on four.  HBM bound: 134 million
// weights with bf16 gradients and their norm take 609 to 620 us, 573 at a copy's rate.
template <int N>
__global__ void __launch_bounds__(kThreads, 4) adamw_kernel(const __grid_constant__ Launch<N> P)
{
    __shared__ Step s;
    __shared__ double warps[kWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    begin_step(P, s);
    constexpr int kSteps = kChunk / kRow;
    Cursor<N> at;
    float keep = 0.0f;
    In32 next;
    bool ahead = false;
    for (unsigned int c = blockIdx.x; c < P.chunks; c += gridDim.x) {
        if (at.go(P, c)) keep = (float)(1.0 - s.lr * P.item[at.t].wd);
        const Item &it = P.item[at.t];
        const long long first = (long long)(c - it.first_chunk) * kChunk, then = first + (long long)gridDim.x * kChunk;
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const long long i = first + k * kRow + threadIdx.x * 4;
            if (first + kChunk <= it.n) {
                In32 in;
                if (ahead) in = next;
                else in = load32<true>(it, i);
                const bool last = k + 1 == kSteps;
                ahead = !last || (c + gridDim.x < at.end && then + kChunk <= it.n);
                if (ahead) next = load32<true>(it, last ? then + threadIdx.x * 4 : i + kRow);
                step32<true>(P, s, it, keep, i, in, sum);
            } else {
                step32<false>(P, s, it, keep, i, load32<false>(it, i), sum);
            }
        }
        if (it.stats) {
            sum = block_sum(sum, warps);
            if (threadIdx.x == 0) P.parts[it.first_part + (c - it.first_chunk)] = sum;
        }
    }
    end_step(P);
}

// ---- moments in 8 bits ------------------------------------------------------------------------------------------------------
// FIELD: the exponent that stands for the block's largest value, 15 (m) or 31 (v).
// Codes are scaled by 2^(E - FIELD) and numbers by 2^(FIELD - E): one product where that is a normal number, else two (of 2^+-(127 - FIELD) and 2^+-(E - 127)), which
// give the same bits.  A block that held what is no number (255) is NaN.
template <int FIELD> __device__ __forceinline__ constexpr float up() { return FIELD == 15 ? 0x1p112f : 0x1p96f; }
template <int FIELD> __device__ __forceinline__ constexpr float down() { return FIELD == 15 ? 0x1p-112f : 0x1p-96f; }
template <int FIELD> __device__ __forceinline__ uint32_t float_of_code(uint32_t codes, int j)
{
    const uint32_t top = __byte_perm(codes, 0, 0x0444 | j << 12);            // the code in the upper byte
    return FIELD == 31 ? top >> 4 : (uint32_t)((int32_t)top >> 4) & 0x87F00000u;
}
template <int FIELD> __device__ __forceinline__ void decode(uint32_t codes, uint32_t e, float (&f)[4])
{
    constexpr uint32_t kBias = 127 - FIELD;
    if (e <= 254 - kBias) {
        const float scale = __uint_as_float((e + kBias) << 23);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = __fmul_rn(__uint_as_float(float_of_code<FIELD>(codes, j)), scale);
    } else {
        const float unit = __uint_as_float(e == 255 ? 0x7FC00000u : e << 23);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = __fmul_rn(__fmul_rn(__uint_as_float(float_of_code<FIELD>(codes, j)), up<FIELD>()), unit);
    }
}
// Exponent of a warp's 128 values; 255 where one of them is no number, or so large (over 3.19e38) that it would round to infinity.
template <bool SIGNED> __device__ __forceinline__ uint32_t exponent_of(const float (&f)[4])
{
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) most = max(most, __float_as_uint(SIGNED ? fabsf(f[j]) : f[j]));
    return min((__reduce_max_sync(0xffffffffu, most) + 0xFFFFFu) >> 23, 255u);
}
// r: what is added below a code, sixteen bits for the upper ones of twenty (and the middle of what they leave).
template <int FIELD> __device__ __forceinline__ uint32_t encode(const float (&f)[4], uint32_t e, const uint32_t (&r)[4])
{
    constexpr uint32_t kTop = 127 + FIELD;
    uint32_t z[4];
    if (e < kTop) {
        const float scale = __uint_as_float((kTop - e) << 23);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = __float_as_uint(__fmul_rn(fabsf(f[j]), scale));
    } else {
        const float inv = __uint_as_float(e >= 254 ? 0x00400000u : (254 - e) << 23);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = __float_as_uint(__fmul_rn(__fmul_rn(fabsf(f[j]), inv), down<FIELD>()));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        z[j] += r[j] * 16 + 8;
        if (FIELD == 31) z[j] = (f[j] > 0.0f ? max(z[j], 0x00100000u) : z[j]) << 4;
        else z[j] = (z[j] << 4 & 0x7FFFFFFFu) | (__float_as_uint(f[j]) & 0x80000000u);
    }
    return __byte_perm(__byte_perm(z[0], z[1], 0x0073), __byte_perm(z[2], z[3], 0x0073), 0x5410);
}

// Four codes from element i on.
__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, long long i, long long n, bool whole)
{
    if (whole) return *reinterpret_cast<const uint32_t *>(p + i);
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) c |= (uint32_t)p[i + j] << (8 * j);
    return c;
}
__device__ __forceinline__ void store_codes(uint8_t *p, long long i, long long n, bool whole, uint32_t c)
{
    if (whole) {
        *reinterpret_cast<uint32_t *>(p + i) = c;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) p[i + j] = (uint8_t)(c >> (8 * j));
}

// The weight's step: the root, the quotient and the sum before it by the fast instructions, within 2^-21 of the formula.  With those that are rounded right 67 million
// weights and the unpacking of their moments took 343 us for 276.
__device__ __forceinline__ float updated_fast(float w, float m, float v, float keep, float a, float rs2, float eps)
{
    float root, inv;
    // (a v below the normal numbers counts as the smallest of them, a NaN stays one)
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(root) : "f"(v), "f"(0x1p-126f));
    asm("sqrt.approx.ftz.f32 %0, %0;" : "+f"(root));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(fmaf(root, rs2, eps)));
    return fmaf(-a, __fmul_rn(m, inv), __fmul_rn(w, keep));
}

// Two rows of weights of a thread, on their way into its own slots in shared memory while those before them are worked on (a slot of each row: W, the gradient, the codes), and
// what of them comes into registers.  The chunks that are not all there come straight from memory.
constexpr int kRows8 = kChunk / kRow, kSlot8 = 16 + 16 + 4 + 4, kStage8 = kRows8 * kSlot8 * kThreads, kStages8 = 2;
static_assert(kRows8 * kRow == kChunk, "a stage is a chunk");
__device__ __forceinline__ void copy_async(uint32_t to, const void *from, int bytes)
{
    if (bytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else if (bytes == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
struct Exponents {
    uint32_t m[kRows8], v[kRows8];
};
// Asks for a chunk from weight `first` on; its exponents.
__device__ __forceinline__ Exponents ask8(const Item &it, long long first, uint32_t stage)
{
    Exponents e;
#pragma unroll
    for (int u = 0; u < kRows8; ++u) {
        const long long i = first + u * kRow + threadIdx.x * 4;
        const uint32_t at = stage + u * (kSlot8 * kThreads);
        copy_async(at + threadIdx.x * 16, it.W + i, 16);
        if (it.g_bf16) copy_async(at + 16 * kThreads + threadIdx.x * 8, static_cast<const __nv_bfloat16 *>(it.dW) + i, 8);
        else copy_async(at + 16 * kThreads + threadIdx.x * 16, static_cast<const float *>(it.dW) + i, 16);
        copy_async(at + 32 * kThreads + threadIdx.x * 4, static_cast<const uint8_t *>(it.m) + i, 4);
        copy_async(at + 36 * kThreads + threadIdx.x * 4, static_cast<const uint8_t *>(it.v) + i, 4);
        e.m[u] = it.m_exp[i / kBlock8];
        e.v[u] = it.v_exp[i / kBlock8];
    }
    return e;
}
struct In8 {
    float w[kRows8][4], g[kRows8][4];
    uint32_t m[kRows8], v[kRows8];
    Exponents e;
};
__device__ __forceinline__ void take8(const Item &it, const uint8_t *stage, In8 &in)
{
#pragma unroll
    for (int u = 0; u < kRows8; ++u) {
        const uint8_t *at = stage + u * (kSlot8 * kThreads);
        const float4 w = *reinterpret_cast<const float4 *>(at + threadIdx.x * 16);
        in.w[u][0] = w.x; in.w[u][1] = w.y; in.w[u][2] = w.z; in.w[u][3] = w.w;
        if (it.g_bf16) {
            const uint2 r = *reinterpret_cast<const uint2 *>(at + 16 * kThreads + threadIdx.x * 8);
            in.g[u][0] = __uint_as_float(r.x << 16); in.g[u][1] = __uint_as_float(r.x & 0xFFFF0000u);
            in.g[u][2] = __uint_as_float(r.y << 16); in.g[u][3] = __uint_as_float(r.y & 0xFFFF0000u);
        } else {
            const float4 r = *reinterpret_cast<const float4 *>(at + 16 * kThreads + threadIdx.x * 16);
            in.g[u][0] = r.x; in.g[u][1] = r.y; in.g[u][2] = r.z; in.g[u][3] = r.w;
        }
        in.m[u] = *reinterpret_cast<const uint32_t *>(at + 32 * kThreads + threadIdx.x * 4);
        in.v[u] = *reinterpret_cast<const uint32_t *>(at + 36 * kThreads + threadIdx.x * 4);
    }
}
__device__ __forceinline__ void load8(const Item &it, long long first, In8 &in)
{
#pragma unroll
    for (int u = 0; u < kRows8; ++u) {
        const long long i = first + u * kRow + threadIdx.x * 4;
        const bool whole = i + 4 <= it.n, any = i / kBlock8 * kBlock8 < it.n;
        load_four(it.W, i, it.n, whole, in.w[u]);
        load_gradient(it, i, whole, in.g[u]);
        in.m[u] = load_codes(static_cast<const uint8_t *>(it.m), i, it.n, whole);
        in.v[u] = load_codes(static_cast<const uint8_t *>(it.v), i, it.n, whole);
        in.e.m[u] = any ? it.m_exp[i / kBlock8] : 0;
        in.e.v[u] = any ? it.v_exp[i / kBlock8] : 0;
    }
}
template <bool FULL, int N> __device__ __forceinline__ void step8(const Launch<N> &P, const Step &s, const Item &it, float keep, long long first, In8 &in, double &sum)
{
#pragma unroll
    for (int u = 0; u < kRows8; ++u) {
        const long long i = first + u * kRow + threadIdx.x * 4;
        const bool whole = FULL || i + 4 <= it.n;
        float m[4], v[4];
        uint32_t rm[4], rv[4];
        decode<15>(in.m[u], in.e.m[u], m);
        decode<31>(in.v[u], in.e.v[u], v);
        // (the index of a weight past 2^32 goes into the hash with all its bits)
        const uint32_t at = (uint32_t)i + (uint32_t)(i >> 32) * 0x9E3779B9u + s.key;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            moments(__fmul_rn(in.g[u][j], s.scale), m[j], v[j], P.b1, P.ob1, P.b2, P.ob2);
            in.w[u][j] = updated_fast(in.w[u][j], m[j], v[j], keep, s.a, s.rs2, P.eps);
            const uint32_t h = mix(at + j);
            rm[j] = h & 0xFFFFu;
            rv[j] = h >> 16;
        }
        store_four(it.W, i, it.n, whole, in.w[u]);
        const uint32_t e1 = exponent_of<true>(m), e2 = exponent_of<false>(v);
        store_codes(static_cast<uint8_t *>(it.m), i, it.n, whole, encode<15>(m, e1, rm));
        store_codes(static_cast<uint8_t *>(it.v), i, it.n, whole, encode<31>(v, e2, rv));
        if ((threadIdx.x & 31) == 0 && (FULL || i < it.n)) {
            it.m_exp[i / kBlock8] = (uint8_t)e1;
            it.v_exp[i / kBlock8] = (uint8_t)e2;
        }
        add_sizes<FULL>(it, i, in.w[u], sum);
    }
}
// Bound by instructions (81 % of the issue slots): 67 million weights with bf16 gradients take 203 to 213 us, their 942 MB alone 144.  88 instructions a weight: the
// update, two decodings, two stochastic roundings and a hash.  The order of chunks is that of the kernel above (with a run of chunks of each block 397 us
// for 303 at the time: all blocks then read from as many places); more blocks an SM have too few registers.
template <int N>
__global__ void __launch_bounds__(kThreads, 4) adamw8_kernel(const __grid_constant__ Launch<N> P)
{
    extern __shared__ __align__(16) uint8_t ring8[];
    __shared__ Step s;
    __shared__ double warps[kWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    Cursor<N> here, there;                               // what is worked on, what is asked for
    Exponents e[kStages8];
    auto ask = [&](unsigned int c, int stage) {
        if (c < P.chunks) {
            there.go(P, c);
            const Item &it = P.item[there.t];
            const long long first = (long long)(c - it.first_chunk) * kChunk;
            if (first + kChunk <= it.n) e[stage] = ask8(it, first, (uint32_t)__cvta_generic_to_shared(ring8) + stage * kStage8);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kStages8; ++k) ask(blockIdx.x + k * gridDim.x, k);
    begin_step(P, s);
    float keep = 0.0f;
    for (unsigned int c0 = blockIdx.x; c0 < P.chunks; c0 += kStages8 * gridDim.x)
#pragma unroll
        for (int k = 0; k < kStages8; ++k) {
            const unsigned int c = c0 + k * gridDim.x;
            if (c >= P.chunks) break;
            if (here.go(P, c)) keep = (float)(1.0 - s.lr * P.item[here.t].wd);
            const Item &it = P.item[here.t];
            const long long first = (long long)(c - it.first_chunk) * kChunk;
            double sum = 0.0;
            In8 in;
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages8 - 1) : "memory");
            if (first + kChunk <= it.n) {
                take8(it, ring8 + k * kStage8, in);
                in.e = e[k];
                ask(c + kStages8 * gridDim.x, k);
                step8<true>(P, s, it, keep, first, in, sum);
            } else {
                ask(c + kStages8 * gridDim.x, k);
                load8(it, first, in);
                step8<false>(P, s, it, keep, first, in, sum);
            }
            if (it.stats) {
                sum = block_sum(sum, warps);
                if (threadIdx.x == 0) P.parts[it.first_part + (c - it.first_chunk)] = sum;
            }
        }
    end_step(P);
}

// What the updated weights of a tensor leave for its next thresholds: one block per tensor.
template <int N>
__global__ void __launch_bounds__(kThreads) adamw_fold_kernel(const __grid_constant__ Launch<N> P)
{
    __shared__ double warps[kWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Item &it = P.item[blockIdx.x];
    if (!it.stats) return;
    const long long parts = (it.n + kChunk - 1) / kChunk;
    double a = 0.0;
#pragma unroll 8
    for (long long i = threadIdx.x; i < parts; i += kThreads) a += P.parts[it.first_part + i];
    a = block_sum(a, warps);
    if (threadIdx.x == 0) {
        it.stats->sum_abs = a;
        it.stats->delta = it.n > 0 ? P.factor * (a / (double)it.n) : 0.0;
        it.stats->status = isfinite(a) ? TWN_OK : TWN_ERR_NONFINITE;
        it.stats->reserved = 0;
    }
}

// ---- moments of 8 bits as numbers ---------------------------------------------------------------------------------------------
struct UnpackItem {
    const uint8_t *m, *v, *m_exp, *v_exp;
    void *m_out, *v_out;
    long long n;
    unsigned int first_chunk;
    int bf16;
};
template <int N> struct UnpackLaunch {
    int count;
    unsigned int chunks;
    UnpackItem item[N];
};
// HBM bound: 67 million weights' moments, 2.02 bytes read and 4 written of each, take 68 us (6 TB/s).
constexpr int kUnpackChunk = 4096;
// Eight codes of a thread: 8 bytes read, 16 or 32 written.
template <int FIELD> __device__ __forceinline__ void unpack_eight(uint2 c, uint32_t e, void *out, bool bf16, long long i)
{
    float a[4], b[4];
    decode<FIELD>(c.x, e, a);
    decode<FIELD>(c.y, e, b);
    if (bf16) {
        uint32_t r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float *f = k < 2 ? a : b;
            const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * (k & 1)], f[2 * (k & 1) + 1]);
            r[k] = *reinterpret_cast<const uint32_t *>(&v);
        }
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(out) + i) = make_uint4(r[0], r[1], r[2], r[3]);
    } else {
        *reinterpret_cast<float4 *>(static_cast<float *>(out) + i) = make_float4(a[0], a[1], a[2], a[3]);
        *reinterpret_cast<float4 *>(static_cast<float *>(out) + i + 4) = make_float4(b[0], b[1], b[2], b[3]);
    }
}
template <int FIELD> __device__ __forceinline__ void unpack_rest(const uint8_t *codes, const uint8_t *exps, void *out, bool bf16, long long i, long long n)
{
    for (long long j = i; j < min(i + 8, n); ++j) {
        float f[4];
        decode<FIELD>(codes[j], exps[j / kBlock8], f);
        if (bf16) static_cast<__nv_bfloat16 *>(out)[j] = __float2bfloat16_rn(f[0]);
        else static_cast<float *>(out)[j] = f[0];
    }
}
template <int FIELD> __device__ __forceinline__ void unpack_chunk(const uint8_t *codes, const uint8_t *exps, void *out, bool bf16, long long first, long long n)
{
    constexpr int U = kUnpackChunk / (8 * kThreads);
    const long long i0 = first + threadIdx.x * 8;
    if (first + kUnpackChunk <= n) {
        uint2 c[U];
        uint32_t e[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = i0 + u * 8 * kThreads;
            c[u] = __ldg(reinterpret_cast<const uint2 *>(codes + i));
            e[u] = __ldg(exps + i / kBlock8);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) unpack_eight<FIELD>(c[u], e[u], out, bf16, i0 + u * 8 * kThreads);
    } else {
        for (int u = 0; u < U; ++u) unpack_rest<FIELD>(codes, exps, out, bf16, i0 + u * 8 * kThreads, n);
    }
}
template <int N>
__global__ void __launch_bounds__(kThreads) adamw8_unpack_kernel(const __grid_constant__ UnpackLaunch<N> P)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (unsigned int c = blockIdx.x; c < P.chunks; c += gridDim.x) {
        int lo = 0;
        for (int hi = P.count; hi - lo > 1;) {
            const int mid = (lo + hi) >> 1;
            if (c >= P.item[mid].first_chunk) lo = mid;
            else hi = mid;
        }
        const UnpackItem &it = P.item[lo];
        const long long first = (long long)(c - it.first_chunk) * kUnpackChunk;
        if (it.m_out) unpack_chunk<15>(it.m, it.m_exp, it.m_out, it.bf16, first, it.n);
        if (it.v_out) unpack_chunk<31>(it.v, it.v_exp, it.v_out, it.bf16, first, it.n);
    }
}

// ---- the norm of all gradients ------------------------------------------------------------------------------------------------
// Squares and sums are fp64: no square leaves its range, and the norm is right to its last bit or nearly.  32 KB of a tensor at a time, all of a thread's loads before the
// first is used (with one load at a time and its sum ResNet-18's norm and update took 76 us for 67).  HBM bound.
struct NormItem {
    const void *dW;
    long long n;
    unsigned int first_chunk;
    int bf16;
};
template <int N> struct NormLaunch {
    int count;
    unsigned int chunks;
    double *parts;
    NormItem item[N];
};
constexpr int kNormLoads = 8, kNormBytes = kNormLoads * 16 * kThreads, kNormBlocksPerSm = 4, kMaxNormParts = kNormBlocksPerSm * 148;

template <int N>
__global__ void __launch_bounds__(kThreads, kNormBlocksPerSm) grad_norm_kernel(const __grid_constant__ NormLaunch<N> P)
{
    __shared__ double warps[kWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double a[4] = {0.0, 0.0, 0.0, 0.0};
    auto add = [&](float g, int k) { a[k] = fma((double)g, (double)g, a[k]); };
    for (unsigned int c = blockIdx.x; c < P.chunks; c += gridDim.x) {
        int lo = 0;
        for (int hi = P.count; hi - lo > 1;) {
            const int mid = (lo + hi) >> 1;
            if (c >= P.item[mid].first_chunk) lo = mid;
            else hi = mid;
        }
        const NormItem &it = P.item[lo];
        const int size = it.bf16 ? 2 : 4;
        const long long first = (long long)(c - it.first_chunk) * kNormBytes;
        const char *const p = static_cast<const char *>(it.dW) + first;
        const int bytes = (int)min((long long)kNormBytes, it.n * size - first), at = threadIdx.x * 16;
        uint4 r[kNormLoads];
        if (bytes == kNormBytes) {
#pragma unroll
            for (int u = 0; u < kNormLoads; ++u) r[u] = __ldg(reinterpret_cast<const uint4 *>(p + at + u * kThreads * 16));
        } else {
#pragma unroll
            for (int u = 0; u < kNormLoads; ++u) {
                const int from = at + u * kThreads * 16;
                r[u] = make_uint4(0u, 0u, 0u, 0u);
                if (from + 16 <= bytes) {
                    r[u] = __ldg(reinterpret_cast<const uint4 *>(p + from));
                } else {
                    for (int j = from; j < bytes; j += size)
                        add(it.bf16 ? __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(p + j)) : *reinterpret_cast<const float *>(p + j), 0);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kNormLoads; ++u) {
            const uint32_t w[4] = {r[u].x, r[u].y, r[u].z, r[u].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (it.bf16) {
                    add(__uint_as_float(w[k] << 16), k);
                    add(__uint_as_float(w[k] & 0xFFFF0000u), k);
                } else {
                    add(__uint_as_float(w[k]), k);
                }
            }
        }
    }
    const double s = block_sum((a[0] + a[2]) + (a[1] + a[3]), warps);
    if (threadIdx.x == 0) P.parts[blockIdx.x] = s;
}
__global__ void __launch_bounds__(kThreads) grad_norm_fold_kernel(const double *parts, int count, double max_norm, float *norm, float *scale)
{
    __shared__ double warps[kWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double a = 0.0;
    for (int i = threadIdx.x; i < count; i += kThreads) a += parts[i];
    a = block_sum(a, warps);
    if (threadIdx.x == 0) {
        // (a norm of finite gradients that is above all numbers of fp32 still clips them)
        const float root = (float)sqrt(a);
        const double r = max_norm / ((isinf(root) ? sqrt(a) : (double)root) + 1e-6);
        if (norm) *norm = root;
        if (scale) *scale = r >= 1.0 ? 1.0f : (float)r;              // a NaN stays one
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------------
bool is_dtype(int d) { return d == TWN_F32 || d == TWN_BF16; }
constexpr long long kMaxN = 1ll << 40;                               // weights of a tensor
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// What a call writes lies apart from all else that it reads or writes.
struct Extents {
    struct Extent {
        uintptr_t begin, end;
        bool written;
    } e[7 * kMaxTensors + 4];
    int n = 0;
    void add(const void *p, long long bytes, bool written)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p && bytes > 0) e[n++] = {at, at + (uintptr_t)bytes, written};
    }
    bool apart()
    {
        std::sort(e, e + n, [](const Extent &a, const Extent &b) { return a.begin < b.begin; });
        uintptr_t any = 0, written = 0;                              // ends of what begins before
        for (int i = 0; i < n; ++i) {
            if (e[i].begin < (e[i].written ? any : written)) return false;
            any = std::max(any, e[i].end);
            if (e[i].written) written = std::max(written, e[i].end);
        }
        return true;
    }
};

bool is_rate(double b) { return b >= 0.0 && b < 1.0; }

struct Hyper {
    double lr, beta1, beta2, eps, factor;
    unsigned long long seed;
    twn_adamw_step_t *step;
    int advance;
    const float *grad_scale, *lr_scale;
};

// The items of a call as those of a launch, checked; TWN_OK or why not.
int add_item(Launch<kMaxTensors> &P, Extents &x, float *W, const void *dW, int g_dtype, void *m, void *v, uint8_t *m_exp, uint8_t *v_exp, int64_t n, double wd,
             twn_stats_t *stats, bool eight, long long *chunks, long long *parts)
{
    TWN_REQUIRE(n >= 0 && n <= kMaxN && is_dtype(g_dtype) && std::isfinite(wd), TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(n == 0 || (W && dW && m && v && (!eight || (m_exp && v_exp))), TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(twn_aligned(W, 16) && twn_aligned(dW, 16) && twn_aligned(m, 16) && twn_aligned(v, 16) && twn_aligned(stats, 8), TWN_ERR_MISALIGNED);
    x.add(W, 4 * n, true);
    x.add(dW, (g_dtype == TWN_BF16 ? 2 : 4) * n, false);
    x.add(m, (eight ? 1 : 4) * n, true);
    x.add(v, (eight ? 1 : 4) * n, true);
    x.add(m_exp, ceil_div(n, kBlock8), true);
    x.add(v_exp, ceil_div(n, kBlock8), true);
    x.add(stats, sizeof(twn_stats_t), true);
    P.item[P.count++] = {W, dW, m, v, m_exp, v_exp, n, wd, stats, (unsigned int)*chunks, (unsigned int)*parts, g_dtype == TWN_BF16};
    *chunks += ceil_div(n, kChunk);
    if (stats) *parts += ceil_div(n, kChunk);
    return *chunks < 1ll << 31 ? TWN_OK : TWN_ERR_TOO_LARGE;
}

template <int N> int launch_update(const Launch<kMaxTensors> &all, bool eight, bool fold, const twn_device_info &dev, cudaStream_t s)
{
    Launch<N> P;
    static_assert(sizeof(Launch<N>) <= 32764, "a launch's parameters");
    P.count = all.count; P.advance = all.advance; P.chunks = all.chunks;
    P.b1 = all.b1; P.ob1 = all.ob1; P.b2 = all.b2; P.ob2 = all.ob2; P.eps = all.eps;
    P.lr = all.lr; P.one_minus_b1 = all.one_minus_b1; P.one_minus_b2 = all.one_minus_b2; P.factor = all.factor;
    P.seed = all.seed; P.step = all.step; P.grad_scale = all.grad_scale; P.lr_scale = all.lr_scale; P.parts = all.parts;
    std::copy(all.item, all.item + std::min(all.count, N), P.item);
    // with nothing to update one block counts the step
    const int grid = (int)std::max(1u, std::min(P.chunks, (unsigned int)dev.sm_count * 4));
    if (eight) {
        static bool done[64] = {false};
        if (!done[dev.ordinal]) TWN_CUDA_OK(cudaFuncSetAttribute(adamw8_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStages8 * kStage8));
        done[dev.ordinal] = true;
    }
    TWN_CUDA_OK(twn_launch_pdl(true, eight ? adamw8_kernel<N> : adamw_kernel<N>, grid, kThreads, eight ? kStages8 * kStage8 : 0, s, P));
    if (fold) TWN_CUDA_OK(twn_launch_pdl(true, adamw_fold_kernel<N>, P.count, kThreads, 0, s, P));
    return TWN_OK;
}

int update(Launch<kMaxTensors> &P, Extents &x, const Hyper &h, bool eight, long long chunks, long long parts, void *workspace, size_t workspace_bytes,
           cudaStream_t s)
{
    if (parts) {
        TWN_REQUIRE(workspace != nullptr && workspace_bytes >= (size_t)parts * sizeof(double), TWN_ERR_WORKSPACE);
        TWN_REQUIRE(twn_aligned(workspace, 256), TWN_ERR_MISALIGNED);
        x.add(workspace, parts * (long long)sizeof(double), true);
    }
    x.add(h.step, sizeof(twn_adamw_step_t), true);
    x.add(h.grad_scale, 4, false);
    x.add(h.lr_scale, 4, false);
    TWN_REQUIRE(x.apart(), TWN_ERR_INVALID_ARG);
    P.advance = h.advance;
    P.chunks = (unsigned int)chunks;
    P.b1 = (float)h.beta1; P.ob1 = (float)(1.0 - h.beta1);
    P.b2 = (float)h.beta2; P.ob2 = (float)(1.0 - h.beta2);
    P.one_minus_b1 = 1.0 - h.beta1; P.one_minus_b2 = 1.0 - h.beta2;
    P.eps = (float)h.eps; P.lr = h.lr; P.factor = h.factor; P.seed = h.seed;
    P.step = h.step; P.grad_scale = h.grad_scale; P.lr_scale = h.lr_scale;
    P.parts = static_cast<double *>(workspace);
    twn_device_info dev;
    const int rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    bool fold = false;
    for (int t = 0; t < P.count; ++t) fold |= P.item[t].stats != nullptr;
    if (P.count <= 1) return launch_update<1>(P, eight, fold, dev, s);
    if (P.count <= 32) return launch_update<32>(P, eight, fold, dev, s);
    return launch_update<kMaxTensors>(P, eight, fold, dev, s);
}

int check(const Hyper &h, const void *items, int count)
{
    TWN_REQUIRE(count >= 0 && count <= kMaxTensors && (count == 0 || items != nullptr), TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(std::isfinite(h.lr) && is_rate(h.beta1) && is_rate(h.beta2) && std::isfinite(h.eps) && (float)h.eps > 0.0f, TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(std::isfinite(h.factor) && h.factor >= 0.0, TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(h.step != nullptr && (h.advance == 0 || h.advance == 1), TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(twn_aligned(h.step, 8) && twn_aligned(h.grad_scale, 4) && twn_aligned(h.lr_scale, 4), TWN_ERR_MISALIGNED);
    return TWN_OK;
}

size_t in_256(size_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

extern "C" size_t twn_adamw_workspace_bytes(const int64_t *n, int count)
{
    if (n == nullptr || count <= 0 || count > kMaxTensors) return 0;
    size_t parts = 0;
    for (int t = 0; t < count; ++t) {
        if (n[t] < 0 || n[t] > kMaxN) return 0;
        parts += (size_t)ceil_div(n[t], kChunk);
    }
    return in_256(parts * sizeof(double));
}

extern "C" int twn_adamw_update_batch(const twn_adamw_item_t *items, int count, double lr, double beta1, double beta2, double eps, double delta_factor,
                                      twn_adamw_step_t *step, int32_t advance, const float *grad_scale, const float *lr_scale, void *workspace,
                                      size_t workspace_bytes, twn_stream_t stream)
{
    const Hyper h = {lr, beta1, beta2, eps, delta_factor, 0, step, advance, grad_scale, lr_scale};
    int rc = check(h, items, count);
    if (rc != TWN_OK) return rc;
    Launch<kMaxTensors> P;
    Extents x;
    P.count = 0;
    long long chunks = 0, parts = 0;
    for (int t = 0; t < count; ++t) {
        const twn_adamw_item_t &it = items[t];
        rc = add_item(P, x, it.W, it.dW, it.g_dtype, it.m, it.v, nullptr, nullptr, it.n, it.weight_decay, it.stats_next, false, &chunks, &parts);
        if (rc != TWN_OK) return rc;
    }
    return update(P, x, h, false, chunks, parts, workspace, workspace_bytes, twn_cu(stream));
}

extern "C" int twn_adamw8_update_batch(const twn_adamw8_item_t *items, int count, double lr, double beta1, double beta2, double eps, double delta_factor,
                                       uint64_t seed, twn_adamw_step_t *step, int32_t advance, const float *grad_scale, const float *lr_scale,
                                       void *workspace, size_t workspace_bytes, twn_stream_t stream)
{
    const Hyper h = {lr, beta1, beta2, eps, delta_factor, seed, step, advance, grad_scale, lr_scale};
    int rc = check(h, items, count);
    if (rc != TWN_OK) return rc;
    Launch<kMaxTensors> P;
    Extents x;
    P.count = 0;
    long long chunks = 0, parts = 0;
    for (int t = 0; t < count; ++t) {
        const twn_adamw8_item_t &it = items[t];
        rc = add_item(P, x, it.W, it.dW, it.g_dtype, it.m, it.v, it.m_exp, it.v_exp, it.n, it.weight_decay, it.stats_next, true, &chunks, &parts);
        if (rc != TWN_OK) return rc;
    }
    return update(P, x, h, true, chunks, parts, workspace, workspace_bytes, twn_cu(stream));
}

extern "C" int twn_adamw8_unpack_batch(const twn_adamw8_states_t *items, int count, twn_stream_t stream)
{
    TWN_REQUIRE(count >= 0 && count <= kMaxTensors && (count == 0 || items != nullptr), TWN_ERR_INVALID_ARG);
    UnpackLaunch<kMaxTensors> P;
    static_assert(sizeof(P) <= 32764, "a launch's parameters");
    Extents x;
    P.count = 0;
    long long chunks = 0;
    for (int t = 0; t < count; ++t) {
        const twn_adamw8_states_t &it = items[t];
        TWN_REQUIRE(it.n >= 0 && it.n <= kMaxN && is_dtype(it.out_dtype), TWN_ERR_INVALID_ARG);
        if (it.n == 0) continue;
        TWN_REQUIRE((!it.m_out || (it.m && it.m_exp)) && (!it.v_out || (it.v && it.v_exp)), TWN_ERR_INVALID_ARG);
        TWN_REQUIRE(twn_aligned(it.m, 16) && twn_aligned(it.v, 16) && twn_aligned(it.m_out, 16) && twn_aligned(it.v_out, 16), TWN_ERR_MISALIGNED);
        for (const void *p : {(const void *)it.m_out, (const void *)it.v_out}) x.add(p, (it.out_dtype == TWN_BF16 ? 2 : 4) * it.n, true);
        if (it.m_out) { x.add(it.m, it.n, false); x.add(it.m_exp, ceil_div(it.n, kBlock8), false); }
        if (it.v_out) { x.add(it.v, it.n, false); x.add(it.v_exp, ceil_div(it.n, kBlock8), false); }
        P.item[P.count++] = {it.m, it.v, it.m_exp, it.v_exp, it.m_out, it.v_out, it.n, (unsigned int)chunks, it.out_dtype == TWN_BF16};
        chunks += ceil_div(it.n, kUnpackChunk);
        TWN_REQUIRE(chunks < 1ll << 31, TWN_ERR_TOO_LARGE);
    }
    TWN_REQUIRE(x.apart(), TWN_ERR_INVALID_ARG);
    if (P.count == 0) return TWN_OK;
    P.chunks = (unsigned int)chunks;
    twn_device_info dev;
    const int rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    const int grid = (int)std::min(P.chunks, (unsigned int)dev.sm_count * 8);
    cudaStream_t s = twn_cu(stream);
    if (P.count <= 32) {
        UnpackLaunch<32> Q;
        Q.count = P.count;
        Q.chunks = P.chunks;
        std::copy(P.item, P.item + P.count, Q.item);
        TWN_CUDA_OK(twn_launch_pdl(true, adamw8_unpack_kernel<32>, grid, kThreads, 0, s, Q));
    } else {
        TWN_CUDA_OK(twn_launch_pdl(true, adamw8_unpack_kernel<kMaxTensors>, grid, kThreads, 0, s, P));
    }
    return TWN_OK;
}

extern "C" size_t twn_grad_norm_workspace_bytes(const int64_t *n, int count)
{
    if (n == nullptr || count <= 0 || count > kMaxTensors) return 0;
    long long chunks = 0;
    for (int t = 0; t < count; ++t) {
        if (n[t] < 0 || n[t] > kMaxN) return 0;
        chunks += ceil_div(4 * n[t], kNormBytes);
    }
    return in_256((size_t)std::max(1ll, std::min<long long>(chunks, kMaxNormParts)) * sizeof(double));
}

extern "C" int twn_grad_norm_batch(const twn_grad_item_t *items, int count, double max_norm, float *norm, float *scale, void *workspace,
                                   size_t workspace_bytes, twn_stream_t stream)
{
    TWN_REQUIRE(count >= 0 && count <= kMaxTensors && (count == 0 || items != nullptr) && max_norm > 0.0 && std::isfinite(max_norm), TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(twn_aligned(norm, 4) && twn_aligned(scale, 4), TWN_ERR_MISALIGNED);
    NormLaunch<kMaxTensors> P;
    Extents x;
    P.count = 0;
    long long chunks = 0;
    for (int t = 0; t < count; ++t) {
        const twn_grad_item_t &it = items[t];
        TWN_REQUIRE(it.n >= 0 && it.n <= kMaxN && is_dtype(it.dtype) && (it.n == 0 || it.dW), TWN_ERR_INVALID_ARG);
        TWN_REQUIRE(twn_aligned(it.dW, 16), TWN_ERR_MISALIGNED);
        if (it.n == 0) continue;
        x.add(it.dW, (it.dtype == TWN_BF16 ? 2 : 4) * it.n, false);
        P.item[P.count++] = {it.dW, it.n, (unsigned int)chunks, it.dtype == TWN_BF16};
        chunks += ceil_div((it.dtype == TWN_BF16 ? 2 : 4) * it.n, kNormBytes);
        TWN_REQUIRE(chunks < 1ll << 31, TWN_ERR_TOO_LARGE);
    }
    const int parts = (int)std::min<long long>(chunks, kMaxNormParts);
    if (parts) {
        TWN_REQUIRE(workspace != nullptr && workspace_bytes >= (size_t)parts * sizeof(double), TWN_ERR_WORKSPACE);
        TWN_REQUIRE(twn_aligned(workspace, 256), TWN_ERR_MISALIGNED);
        x.add(workspace, parts * (long long)sizeof(double), true);
    }
    x.add(norm, 4, true);
    x.add(scale, 4, true);
    TWN_REQUIRE(x.apart(), TWN_ERR_INVALID_ARG);
    twn_device_info dev;
    const int rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    P.chunks = (unsigned int)chunks;
    P.parts = static_cast<double *>(workspace);
    cudaStream_t s = twn_cu(stream);
    if (parts) {
        if (P.count <= 32) {
            NormLaunch<32> Q;
            Q.count = P.count;
            Q.chunks = P.chunks;
            Q.parts = P.parts;
            std::copy(P.item, P.item + P.count, Q.item);
            TWN_CUDA_OK(twn_launch_pdl(true, grad_norm_kernel<32>, parts, kThreads, 0, s, Q));
        } else {
            TWN_CUDA_OK(twn_launch_pdl(true, grad_norm_kernel<kMaxTensors>, parts, kThreads, 0, s, P));
        }
    }
    TWN_CUDA_OK(twn_launch_pdl(true, grad_norm_fold_kernel, 1, kThreads, 0, s, P.parts, parts, max_norm, norm, scale));
    return TWN_OK;
}
