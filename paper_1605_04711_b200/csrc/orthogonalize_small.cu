// Orthogonalised updates of small matrices (up to 128 x 8192): all steps in one launch, a cluster of eight blocks a matrix.
//
// Fifteen products of a matrix of 64 rows are fifteen launches of almost nothing, 7 us each.  With few rows there is another way:
// every step multiplies X from the left by a polynomial of its Gram matrix, so with A = X X^T (m x m)
//   B = a I + b A + c A^2,   Q <- B Q,   A <- (B A) B      and at the end   O = Q X0
// X0 itself is read twice, and the steps are products of m x m matrices in one SM's shared and tensor memory.
//
// Rounding.  A small singular value s of X0 is an eigenvalue s^2 of A, so here A has to have the digits: the Gram matrix is summed from
// bf16 parts of G (three of an fp32 element, all 24 bits; six products, those with a lower part in sums of their own, the others
// taken over into fp32 registers every 64 columns), everything after it from two fp16 parts (22 bits, three products), in fp32.  Where X0 has low rank, Q is 485 times the identity nearly
// everywhere, and Q X0 a difference of large terms.  The multiples of the identity are therefore kept apart:
//   B = a I + B',  Q = a^k I + Q',   B' = b A + c A^2,  T = a A + B' A,  A <- a T + T B',  Q' <- a Q' + a^k B' + B' Q',
//   O = a^steps X0 + Q' X0
// and added in fp32 after the product: the tensor core's sums lose up to a unit in the last place with every addition, all the same
// way, so they are given few and small ones (the products of lower parts first, then eight additions).  With whole matrices a
// matrix of rank one was 1.7e-3 off, with the terms put into the accumulators ahead 1.6e-3.  An eigenvalue that rounding has made negative grows as a small positive one does, by a^2 = 11.9 a step, 1e-7 to
// 0.02 in five; from about eight steps on it would run away, so more than five steps go the other way (orthogonalize.cu).
//
// Range.  The Gram matrix is summed before the norm, its trace, is known.  Where that leaves the range in which fp32 keeps its
// digits, it is summed again from G times a power of two, that of the trace where it says how large G is (second_scale).
// X0 of a G below eps has a norm d = |G|_F / eps below 1, however small: the last product is taken with G over its own norm, and its
// result times d.
//
// What bounds it: 14 dependent products of 128 x 128 x 128 (three MMA passes, 0.8 us each) with the elements' way through registers
// between them (about as long), two passes over the matrix by eight SMs, and four cluster barriers.
#include <algorithm>
#include <cmath>

#include <cuda_fp16.h>

#include "orthogonalize.cuh"
#include "tc_ptx.cuh"

namespace {

using namespace twn_detail;

constexpr int kThreads = 512;                // sixteen warps: each has 32 rows and 32 columns of a matrix
constexpr int kQuads = 128 * 64 / 4 / kThreads;
constexpr int kCluster = 8;
constexpr uint32_t kHalfMatrix = 32 * 1024, kMatrix = 2 * kHalfMatrix;      // 128 x 128 fp16; its upper and lower parts
constexpr float kScaleA = 4096.0f, kScaleB = 1024.0f, kScaleT = 4096.0f, kScaleQ = 64.0f, kScaleX = 256.0f;
// columns of tensor memory: A, then T, as they are; a product (A A, B' Q', T B'); B' A; Q' as it is
constexpr uint32_t kColA = 0, kColS = 128, kColT = 256, kColQ = 384;

struct __align__(1024) SmallSmem {
    uint8_t mat[3][kMatrix];                 // A or T, B, Q: each as rows of 64 elements in the 128-byte swizzle, two blocks a part
    unsigned long long bar[2];
    uint32_t tmem_base;
    volatile int abort_flag;
    double red[kThreads / 32];
    // what block 0 says: 1 / max(norm, eps) for X0 = G pre * factor, 1 / norm, and norm / max(norm, eps); whether to sum again with pre
    float factor, by_norm, below, pre;
    int again;
};

__device__ __forceinline__ uint32_t at_block(uint32_t addr, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ float4 ld_cluster(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster(uint32_t a, float4 v)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void whole_cluster()
{
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// fp16 operands, fp32 sums
__host__ __device__ constexpr uint32_t idesc_f16(int N, bool b_mn) { return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(N >> 3) << 17) | (8u << 24); }

// Byte of element (r, c) in rows of 64 16-bit elements, 128 bytes, swizzled.
__device__ __forceinline__ uint32_t swizzled(int r, int c) { return (uint32_t)(r * 128 + ((((c >> 3) ^ r) & 7) << 4) + (c & 7) * 2); }

__device__ __forceinline__ uint32_t half_pair(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 from_half_pair(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
// Two parts of two elements.
__device__ __forceinline__ void two_parts(float a, float b, uint32_t &hi, uint32_t &lo)
{
    hi = half_pair(a, b);
    const float2 h = from_half_pair(hi);
    lo = half_pair(a - h.x, b - h.y);
}

// Four elements of G from row `row` (of its own shape) and column `col` on, zeros past its end; with UPDATE the momentum is
// updated on the way.
enum { kF32, kBf16, kMuon };
template <int KIND, bool UPDATE> __device__ __forceinline__ float4 four(const NsSource &it, const NsSmallParams &P, int row, int col, int rows, int cols, bool vec)
{
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (row < rows && col < cols) {
        const int i = row * cols + col, left = cols - col;
        if (KIND == kMuon) {
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (vec) {
                const float4 a = *reinterpret_cast<const float4 *>(it.V + i), b = *reinterpret_cast<const float4 *>(it.dW + i);
                v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
                d[0] = b.x; d[1] = b.y; d[2] = b.z; d[3] = b.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < left) { v[j] = it.V[i + j]; d[j] = it.dW[i + j]; }
            }
            if (UPDATE) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = __fadd_rn(__fmul_rn(P.momentum, v[j]), d[j]);
                if (vec) {
                    *reinterpret_cast<float4 *>(it.V + i) = make_float4(v[0], v[1], v[2], v[3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < left) it.V[i + j] = v[j];
                }
            }
            if (P.look_ahead)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = __fadd_rn(d[j], __fmul_rn(P.momentum, v[j]));
        } else if (KIND == kBf16) {
            const uint16_t *g = static_cast<const uint16_t *>(it.G) + i;
            if (vec) {
                const uint2 w = *reinterpret_cast<const uint2 *>(g);
                v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
                v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < left) v[j] = __uint_as_float((uint32_t)g[j] << 16);
            }
        } else {
            const float *g = static_cast<const float *>(it.G) + i;
            if (vec) {
                const float4 a = *reinterpret_cast<const float4 *>(g);
                v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < left) v[j] = g[j];
            }
        }
    }
    return make_float4(v[0], v[1], v[2], v[3]);
}
// Place of a thread's quad i of the 64 columns of X from 64 b on, in G's own shape and in the tile: wide matrices have 128 rows of 64,
// tall ones 64 rows of 128, which are two blocks.
struct Quad {
    int row, col;                // in G
    uint32_t at;                 // in a part of the tile
};
__device__ __forceinline__ Quad quad_of(bool tall, int b, int i)
{
    const int tid = threadIdx.x;
    Quad q;
    if (tall) {
        const int c = 4 * (tid & 31), r = (tid >> 5) + (kThreads / 32) * i;
        q.row = 64 * b + r;
        q.col = c;
        q.at = (uint32_t)(c >> 6) * 8192 + swizzled(r, c & 63);
    } else {
        const int c = 4 * (tid & 15), r = (tid >> 4) + (kThreads / 16) * i;
        q.row = r;
        q.col = 64 * b + c;
        q.at = swizzled(r, c);
    }
    return q;
}

// D = P R^T (three products of two parts each, the small ones first) of two matrices of mm x mm in shared memory, by the calling
// thread.
__device__ __forceinline__ void product(uint32_t d, uint32_t p, uint32_t r, int mm)
{
    const uint32_t idesc = idesc_f16(mm, false);
#pragma unroll
    for (int combo = 0; combo < 3; ++combo) {
        const uint64_t a = smem_desc_sw128(p + (combo == 1 ? kHalfMatrix : 0)), b = smem_desc_sw128(r + (combo == 0 ? kHalfMatrix : 0));
        for (int k = 0; k < mm / 16; ++k) {
            const uint64_t off = (uint64_t)((k >> 2) * (16384 >> 4) + 2 * (k & 3));
            mma(d, a + off, b + off, idesc, combo + k > 0);
        }
    }
}

// A row's 32 elements from column c on as the two parts of a matrix in shared memory (and in `copy`, of the same layout).
__device__ __forceinline__ void write_parts(uint8_t *mat, int r, int c, const float (&v)[32], uint8_t *copy = nullptr)
{
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) two_parts(v[8 * p + 2 * j], v[8 * p + 2 * j + 1], h[j], l[j]);
        const uint32_t at = (uint32_t)((c + 8 * p) >> 6) * 16384 + swizzled(r, (c + 8 * p) & 63);
        const uint4 hv = make_uint4(h[0], h[1], h[2], h[3]), lv = make_uint4(l[0], l[1], l[2], l[3]);
        *reinterpret_cast<uint4 *>(mat + at) = hv;
        *reinterpret_cast<uint4 *>(mat + kHalfMatrix + at) = lv;
        if (copy) {
            *reinterpret_cast<uint4 *>(copy + at) = hv;
            *reinterpret_cast<uint4 *>(copy + kHalfMatrix + at) = lv;
        }
    }
}
__device__ __forceinline__ void tmem_put32(uint32_t taddr, const float (&v)[32])
{
    uint32_t w[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) w[j] = __float_as_uint(v[j]);
    tmem_st32(taddr, w);
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_row32(uint32_t taddr, float (&v)[32])
{
    uint32_t w[32];
    tmem_ld32(taddr, w);
    tmem_wait_ld(w);
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(w[j]);
}

__device__ __forceinline__ void tmem_row16(uint32_t taddr, float (&v)[16])
{
    uint32_t w[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]), "=r"(w[8]), "=r"(w[9]),
                   "=r"(w[10]), "=r"(w[11]), "=r"(w[12]), "=r"(w[13]), "=r"(w[14]), "=r"(w[15])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3]), "+r"(w[4]), "+r"(w[5]), "+r"(w[6]), "+r"(w[7]), "+r"(w[8]), "+r"(w[9]),
                   "+r"(w[10]), "+r"(w[11]), "+r"(w[12]), "+r"(w[13]), "+r"(w[14]), "+r"(w[15])
                 :: "memory");
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(w[j]);
}

// What G is multiplied by before its Gram matrix is summed again, the trace of the first sum being finite or not, at most 1e30 or not.
// From 1e-30 on (of up to 2^20 squares those that fell below fp32, 1e-38 each, are less than a hundredth) and where it is finite the trace
// gives it: 2^-h for a trace of 2^2h, 1 to 4 the second time.  Below, G has a norm under 1.1e-15 and 2^100 brings its trace, 2e-90 at
// least for one denormal element, to 3e-30 at least and 2e30 at most; above, its elements are 1e16 at least in all, and 2^-100 leaves
// 2e-22 to 1e23.  (2^100 for every trace below 1e-20 took a row's 2.1e-22 beyond fp32.)
__device__ __forceinline__ float second_scale(double trace)
{
    if (!isfinite(trace)) return 0x1p-100f;
    if (trace < 1e-30) return 0x1p100f;
    return (float)ldexp(1.0, -(ilogb(trace) >> 1));
}

template <int KIND> __global__ void __launch_bounds__(kThreads, 1) ns_small_kernel(const __grid_constant__ NsSmallParams P)
{
    extern __shared__ uint8_t smem_raw[];
    SmallSmem *sm = reinterpret_cast<SmallSmem *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    volatile int *abort_flag = &sm->abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)(blockIdx.x % kCluster);
    const NsSource &it = P.item[blockIdx.x / kCluster].src;
    uint8_t *const scratch = reinterpret_cast<uint8_t *>(P.item[blockIdx.x / kCluster].scratch);
    if (tid == 0) {
        mbar_init(&sm->bar[0], 1);
        mbar_init(&sm->bar[1], 1);
        sm->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm->tmem_base)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm->tmem_base;
    pdl_begin();

    uint32_t phase[2] = {0u, 0u};
    auto wait = [&](int b) {
        mbar_wait_warp(&sm->bar[b], phase[b], abort_flag, P.status, 0);
        phase[b] ^= 1u;
        tc_fence_after();
    };
    // what the threads have written to shared memory is there for the tensor core
    auto ready = [&]() {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    };
    const bool tall = it.tall != 0;
    const int blocks = (it.n + 63) >> 6;                 // of 64 columns of X; this block has every eighth
    const int mine = rank < blocks ? (blocks - rank + kCluster - 1) / kCluster : 0;
    const int rows = tall ? it.n : it.m, cols = tall ? it.m : it.n;      // of G
    const bool vec = it.vec_in && (cols & 3) == 0;
    // rows and columns that are worked on (of the others nothing that is used depends), this thread's row and columns
    const int mm = (it.m + 15) & ~15, q = warp & 3, row = 32 * q + lane, c = 32 * (warp >> 2);
    const bool in = 32 * q < mm && c < mm;
    const uint32_t t_row = tmem + ((uint32_t)(32 * q) << 16);

    // ---- Gram matrix, its trace ------------------------------------------------------------------------------------------
    float pre = 1.0f, factor = 0.0f, by_norm = 0.0f, below = 1.0f;
    constexpr int planes = KIND == kBf16 ? 1 : 3;
#pragma unroll 1
    for (int attempt = 0; attempt < 2; ++attempt) {
        float4 next[kQuads];
        auto fetch = [&](int b) {
#pragma unroll
            for (int i = 0; i < kQuads; ++i) {
                const Quad at = quad_of(tall, b, i);
                next[i] = attempt == 0 ? four<KIND, true>(it, P, at.row, at.col, rows, cols, vec) : four<KIND, false>(it, P, at.row, at.col, rows, cols, vec);
            }
        };
        float total[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) total[j] = 0.0f;
        // the sums of a tile, of 64 columns of X, when its products are done
        auto take = [&](int s) {
            wait(s);
            if (!in) return;
            float v[32];
            tmem_row32(t_row + (s ? kColQ : kColS) + c, v);
#pragma unroll
            for (int j = 0; j < 32; ++j) total[j] += v[j];
        };
        if (mine > 0) fetch(rank);
#pragma unroll 1
        for (int k = 0; k < mine; ++k) {
            const int s = k & 1;
            uint8_t *const tile = sm->mat[0] + s * 3 * 16384;      // planes of 16 KB
            if (k >= 2) take(s);
#pragma unroll
            for (int i = 0; i < kQuads; ++i) {
                const Quad at = quad_of(tall, 0, i);
                if ((tall ? at.col : at.row) >= mm) continue;
                const float f[4] = {next[i].x * pre, next[i].y * pre, next[i].z * pre, next[i].w * pre};
                float rest[4] = {f[0], f[1], f[2], f[3]};
#pragma unroll
                for (int p = 0; p < planes; ++p) {
                    const uint2 w = make_uint2(pack_bf16x2(rest[0], rest[1]), pack_bf16x2(rest[2], rest[3]));
                    *reinterpret_cast<uint2 *>(tile + p * 16384 + at.at) = w;
                    rest[0] -= __uint_as_float(w.x << 16); rest[1] -= __uint_as_float(w.x & 0xFFFF0000u);
                    rest[2] -= __uint_as_float(w.y << 16); rest[3] -= __uint_as_float(w.y & 0xFFFF0000u);
                }
            }
            if (k + 1 < mine) fetch(rank + (k + 1) * kCluster);
            ready();
            if (warp == 0 && elect_one()) {
                const uint32_t base = smem_u32(tile);
                const uint32_t idesc = tall ? make_idesc_mn(128, mm) : make_idesc(128, mm);
                // the product of the upper parts, and apart from it, in sums of their own, those with a lower one
                for (int o = 0; o < (planes == 1 ? 1 : 6); ++o) {
                    const int pa = o == 2 || o == 5 ? 1 : o == 4 ? 2 : 0, pb = o == 1 || o == 5 ? 1 : o == 3 ? 2 : 0;
                    const uint32_t a = base + pa * 16384, b = base + pb * 16384;
                    const uint64_t da = tall ? smem_desc_mn_sw128(a, 8192) : smem_desc_sw128(a), db = tall ? smem_desc_mn_sw128(b, 8192) : smem_desc_sw128(b);
                    const uint64_t step = tall ? 128 : 2;
                    for (int j = 0; j < 4; ++j) mma(tmem + (o ? kColT : s ? kColQ : kColS), da + j * step, db + j * step, idesc, o ? k + o + j > 1 : j > 0);
                }
                tc_commit(&sm->bar[s]);
            }
            __syncwarp();
        }
        for (int k = max(0, mine - 2); k < mine; ++k) take(k & 1);
        // this block's sums to shared memory (behind the tiles), row by row
        float *const sums = reinterpret_cast<float *>(sm->mat[2]);
        if (in) {
            float v[32];
            if (mine > 0 && planes > 1) {
                tmem_row32(t_row + kColT + c, v);
#pragma unroll
                for (int j = 0; j < 32; ++j) total[j] += v[j];
            }
            // 16-byte pieces exchanged by the row, so that a warp's writes spread over the banks
#pragma unroll
            for (int p = 0; p < 8; ++p)
                *reinterpret_cast<float4 *>(sums + row * 128 + ((((c >> 2) + p) ^ lane) & 31) * 4) = make_float4(total[4 * p], total[4 * p + 1], total[4 * p + 2], total[4 * p + 3]);
        }
        tc_fence_before();
        whole_cluster();
        // an eighth of the rows each, the blocks' sums in their order, to block 0
        for (int i = tid; i < mm / kCluster * 32; i += kThreads) {
            const int r = mm / kCluster * rank + (i >> 5);
            if (4 * (i & 31) >= mm) continue;
            const uint32_t at = (uint32_t)(r * 512 + (((i & 31) ^ r) & 31) * 16);
            float4 part[kCluster];
#pragma unroll
            for (int g = 0; g < kCluster; ++g) part[g] = ld_cluster(at_block(smem_u32(sums), (uint32_t)g) + at);
            float4 v = part[0];
#pragma unroll
            for (int g = 1; g < kCluster; ++g) { v.x += part[g].x; v.y += part[g].y; v.z += part[g].z; v.w += part[g].w; }
            st_cluster(at_block(smem_u32(sm->mat[1]), 0) + at, v);
        }
        whole_cluster();
        if (rank == 0) {
            const float *const gram = reinterpret_cast<const float *>(sm->mat[1]);
            double d = 0.0;
            if (tid < mm) d = gram[tid * 128 + (((tid >> 2) ^ tid) & 31) * 4 + (tid & 3)];
            for (int o = 16; o > 0; o >>= 1) d += __shfl_down_sync(0xffffffffu, d, o);
            if (lane == 0) sm->red[warp] = d;
            __syncthreads();
            if (tid == 0) {
                const double trace = (sm->red[0] + sm->red[1]) + (sm->red[2] + sm->red[3]);
                const bool finite = isfinite(trace);
                const bool far = !finite || trace > 1e30 || trace < 1e-20;
                sm->again = attempt == 0 && far;
                sm->pre = second_scale(trace);
                const double scaled = sqrt(trace), least = (double)P.eps * (double)pre;
                sm->factor = !finite ? __uint_as_float(0x7FC00000u) : trace == 0.0 ? 0.0f : (float)(1.0 / (scaled > least ? scaled : least));
                sm->by_norm = finite && scaled < least && trace != 0.0 ? (float)(1.0 / scaled) : sm->factor;
                sm->below = finite && scaled < least ? (float)(scaled / least) : 1.0f;
                if (!sm->again && !finite && P.status) atomicMin(P.status, (int)TWN_ERR_NONFINITE);
            }
        }
        whole_cluster();
        const bool again = ld_cluster_u32(at_block(smem_u32(&sm->again), 0)) != 0;
        factor = __uint_as_float(ld_cluster_u32(at_block(smem_u32(&sm->factor), 0)));
        by_norm = __uint_as_float(ld_cluster_u32(at_block(smem_u32(&sm->by_norm), 0)));
        below = __uint_as_float(ld_cluster_u32(at_block(smem_u32(&sm->below), 0)));
        if (!again) break;
        pre = __uint_as_float(ld_cluster_u32(at_block(smem_u32(&sm->pre), 0)));
        whole_cluster();                                 // all have read it
    }

    // ---- the steps, in block 0 -------------------------------------------------------------------------------------------------
    if (rank == 0) {
        {
            const float *const gram = reinterpret_cast<const float *>(sm->mat[1]);
            if (in) {
                float v[32], w[32];
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                    const float4 x = *reinterpret_cast<const float4 *>(gram + row * 128 + ((((c >> 2) + p) ^ lane) & 31) * 4);
                    v[4 * p] = x.x; v[4 * p + 1] = x.y; v[4 * p + 2] = x.z; v[4 * p + 3] = x.w;
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    v[j] = v[j] * factor * factor;
                    w[j] = v[j];
                    v[j] *= kScaleA;
                }
                tmem_put32(t_row + kColA + c, w);
                write_parts(sm->mat[0], row, c, v);
            }
        }
        float power = 1.0f;                              // a^step
#pragma unroll 1
        for (int step = 0; step < P.steps; ++step, power *= kNsA) {
            const bool last = step + 1 == P.steps;
            ready();
            if (warp == 0 && elect_one()) {
                product(tmem + kColS, smem_u32(sm->mat[0]), smem_u32(sm->mat[0]), mm);
                tc_commit(&sm->bar[0]);
            }
            __syncwarp();
            wait(0);
            // B' = b A + c A A; of Q' what it has beside the product
            if (in) {
                float a[32], v[32];
                tmem_row32(t_row + kColA + c, a);
                tmem_row32(t_row + kColS + c, v);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = fmaf(kNsC / (kScaleA * kScaleA), v[j], kNsB * a[j]);
                if (step == 0) {
                    tmem_put32(t_row + kColQ + c, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) a[j] = v[j] * kScaleQ;
                    write_parts(sm->mat[2], row, c, a, last ? scratch : nullptr);
                } else {
                    tmem_row32(t_row + kColQ + c, a);
#pragma unroll
                    for (int j = 0; j < 32; ++j) a[j] = fmaf(kNsA, a[j], power * v[j]);
                    tmem_put32(t_row + kColQ + c, a);
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= kScaleB;
                write_parts(sm->mat[1], row, c, v);
            }
            if (last && step == 0) break;
            ready();
            if (warp == 0 && elect_one()) {
                if (!last) product(tmem + kColT, smem_u32(sm->mat[1]), smem_u32(sm->mat[0]), mm);
                if (step > 0) product(tmem + kColS, smem_u32(sm->mat[1]), smem_u32(sm->mat[2]), mm);
                tc_commit(&sm->bar[0]);
            }
            __syncwarp();
            wait(0);
            // T = a A + B' A, Q'
            if (in) {
                float a[32], v[32];
                if (!last) {
                    tmem_row32(t_row + kColA + c, a);
                    tmem_row32(t_row + kColT + c, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = fmaf(1.0f / (kScaleB * kScaleA), v[j], kNsA * a[j]);
                    tmem_put32(t_row + kColA + c, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] *= kScaleT;
                    write_parts(sm->mat[0], row, c, v);
                }
                if (step > 0) {
                    tmem_row32(t_row + kColQ + c, a);
                    tmem_row32(t_row + kColS + c, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) a[j] = fmaf(1.0f / (kScaleB * kScaleQ), v[j], a[j]);
                    if (!last) tmem_put32(t_row + kColQ + c, a);
#pragma unroll
                    for (int j = 0; j < 32; ++j) a[j] *= kScaleQ;
                    write_parts(sm->mat[2], row, c, a, last ? scratch : nullptr);
                }
            }
            if (last) break;
            ready();
            if (warp == 0 && elect_one()) {
                product(tmem + kColS, smem_u32(sm->mat[0]), smem_u32(sm->mat[1]), mm);
                tc_commit(&sm->bar[0]);
            }
            __syncwarp();
            wait(0);
            // A = a T + T B'
            if (in) {
                float a[32], v[32];
                tmem_row32(t_row + kColA + c, a);
                tmem_row32(t_row + kColS + c, v);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = fmaf(1.0f / (kScaleT * kScaleB), v[j], kNsA * a[j]);
                tmem_put32(t_row + kColA + c, v);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= kScaleA;
                write_parts(sm->mat[0], row, c, v);
            }
        }
    }
    tc_fence_before();
    whole_cluster();
    tc_fence_after();

    // ---- O = Q X0 ----------------------------------------------------------------------------------------------------------
    if (rank != 0)
        for (int i = tid; i < 2 * mm * (mm / 8); i += kThreads) {
            const int piece = i % (mm / 8), r = i / (mm / 8) % mm, part = i / (mm / 8) / mm;
            const uint32_t at = (uint32_t)part * kHalfMatrix + (uint32_t)(piece >> 3) * 16384 + swizzled(r, 8 * (piece & 7));
            *reinterpret_cast<uint4 *>(sm->mat[2] + at) = __ldcg(reinterpret_cast<const uint4 *>(scratch + at));
        }
    const float x_scale = by_norm * kScaleX, unscale = 1.0f / (kScaleQ * kScaleX), out_scale = below * it.out_scale;
    float power = kScaleQ;                               // a^steps, beside the product
    for (int k = 0; k < P.steps; ++k) power *= kNsA;
    {
        float4 next[kQuads];
        auto fetch = [&](int b) {
#pragma unroll
            for (int i = 0; i < kQuads; ++i) {
                const Quad at = quad_of(tall, b, i);
                next[i] = four<KIND, false>(it, P, at.row, at.col, rows, cols, vec);
            }
        };
        if (mine > 0) fetch(rank);
#pragma unroll 1
        for (int k = 0; k <= mine; ++k) {
            // tile k to the tensor core, then the result of tile k - 1 from it
            if (k < mine) {
                uint8_t *const tile = sm->mat[0] + (k & 1) * 32768;
#pragma unroll
                for (int i = 0; i < kQuads; ++i) {
                    const Quad at = quad_of(tall, 0, i);
                    if ((tall ? at.col : at.row) >= mm) continue;
                    uint32_t h[2], l[2];
                    two_parts(next[i].x * pre * x_scale, next[i].y * pre * x_scale, h[0], l[0]);
                    two_parts(next[i].z * pre * x_scale, next[i].w * pre * x_scale, h[1], l[1]);
                    *reinterpret_cast<uint2 *>(tile + at.at) = make_uint2(h[0], h[1]);
                    *reinterpret_cast<uint2 *>(tile + 16384 + at.at) = make_uint2(l[0], l[1]);
                }
                if (k + 1 < mine) fetch(rank + (k + 1) * kCluster);
                ready();
                if (warp == 0 && elect_one()) {
                    const uint32_t idesc = idesc_f16(64, !tall);
                    const uint32_t qa = smem_u32(sm->mat[2]), xb = smem_u32(tile);
                    for (int combo = 0; combo < 3; ++combo) {
                        const uint64_t a = smem_desc_sw128(qa + (combo == 1 ? kHalfMatrix : 0));
                        const uint32_t x = xb + (combo == 0 ? 16384 : 0);
                        const uint64_t b = tall ? smem_desc_sw128(x) : smem_desc_mn_sw128(x, 8192);
                        for (int j = 0; j < mm / 16; ++j) {
                            const uint64_t a_off = (uint64_t)((j >> 2) * (16384 >> 4) + 2 * (j & 3));
                            const uint64_t b_off = tall ? (uint64_t)((j >> 2) * (8192 >> 4) + 2 * (j & 3)) : (uint64_t)(128 * j);
                            mma(tmem + 64 * (k & 1), a + a_off, b + b_off, idesc, combo + j > 0);
                        }
                    }
                    tc_commit(&sm->bar[k & 1]);
                }
                __syncwarp();
            }
            if (k == 0) continue;
            const int done = k - 1, b = rank + done * kCluster;
            wait(done & 1);
            // a thread has 16 of the tile's 64 columns
            const int part = 16 * (warp >> 2), c0 = 64 * b + part;
            float d[16];
            tmem_row16(t_row + 64 * (done & 1) + part, d);
            tc_fence_before();
            if (row < it.m) {
                float v[16];
                {
                    const uint8_t *const tile = sm->mat[0] + (done & 1) * 32768;
                    if (tall) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const uint32_t at = (uint32_t)(row >> 6) * 8192 + swizzled(part + j, row & 63);
                            v[j] = __half2float(*reinterpret_cast<const __half *>(tile + at)) + __half2float(*reinterpret_cast<const __half *>(tile + 16384 + at));
                        }
                    } else {
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const uint32_t at = swizzled(row, part + 8 * p);
                            const uint4 h = *reinterpret_cast<const uint4 *>(tile + at), l = *reinterpret_cast<const uint4 *>(tile + 16384 + at);
                            const uint32_t hs[4] = {h.x, h.y, h.z, h.w}, ls[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float2 x = from_half_pair(hs[j]), y = from_half_pair(ls[j]);
                                v[8 * p + 2 * j] = x.x + y.x;
                                v[8 * p + 2 * j + 1] = x.y + y.y;
                            }
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = fmaf(power, v[j], d[j]) * unscale * out_scale;
                if (!tall && it.vec_out) {
#pragma unroll
                    for (int j = 0; j < 16; j += 8) {
                        if (c0 + j >= it.n) break;
                        const long long at = (long long)row * it.n + c0 + j;
                        if (it.o_bf16) {
                            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(it.O) + at) =
                                make_uint4(pack_bf16x2(v[j], v[j + 1]), pack_bf16x2(v[j + 2], v[j + 3]), pack_bf16x2(v[j + 4], v[j + 5]), pack_bf16x2(v[j + 6], v[j + 7]));
                        } else {
                            float4 *o = reinterpret_cast<float4 *>(static_cast<float *>(it.O) + at);
                            o[0] = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                            o[1] = make_float4(v[j + 4], v[j + 5], v[j + 6], v[j + 7]);
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (c0 + j >= it.n) break;
                        const long long at = tall ? (long long)(c0 + j) * it.m + row : (long long)row * it.n + c0 + j;
                        if (it.o_bf16) static_cast<__nv_bfloat16 *>(it.O)[at] = __float2bfloat16_rn(v[j]);
                        else static_cast<float *>(it.O)[at] = v[j];
                    }
                }
            }
            __syncthreads();                             // the tile has been read
        }
    }

    tc_fence_before();
    __syncthreads();
    if (sm->abort_flag) {
        // products in flight end well within this
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

}  // namespace

template <int KIND> static int launch(const NsSmallParams &all, const twn_device_info &dev, cudaStream_t s)
{
    NsSmallParams P = all;
    P.count = 0;
    for (int t = 0; t < all.count; ++t) {
        const NsSource &it = all.item[t].src;
        if ((it.V ? kMuon : it.g_bf16 ? kBf16 : kF32) == KIND) P.item[P.count++] = all.item[t];
    }
    if (P.count == 0) return TWN_OK;
    static bool done[64] = {false};
    const int smem = (int)sizeof(SmallSmem) + 1024;
    if (!done[dev.ordinal]) {
        TWN_CUDA_OK(cudaFuncSetAttribute(ns_small_kernel<KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        done[dev.ordinal] = true;
    }
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(P.count * kCluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    TWN_CUDA_OK(cudaLaunchKernelEx(&cfg, ns_small_kernel<KIND>, P));
    return TWN_OK;
}

int twn_detail::ns_small(const NsSmallParams &P, cudaStream_t s)
{
    twn_device_info dev;
    int rc = twn_current_device(&dev);
    if (rc == TWN_OK) rc = launch<kF32>(P, dev, s);
    if (rc == TWN_OK) rc = launch<kBf16>(P, dev, s);
    if (rc == TWN_OK) rc = launch<kMuon>(P, dev, s);
    return rc;
}
