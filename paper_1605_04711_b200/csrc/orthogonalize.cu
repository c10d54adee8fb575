// Orthogonalised updates: Newton-Schulz steps that bring the singular values of an update matrix near 1 (the Muon
// optimiser's rule), on tcgen05.
//
//   X = G / max(|G|_F, eps), the shorter side m as rows (transposed where G is tall), n columns; then `steps` times
//   A = X X^T,   B = b A + c A^2,   X = a X + B X          (a, b, c) = (3.4445, -4.7750, 2.0315)
//
// Rounding.  The products take fp16 operands and sum in fp32: everything here is at most about 1.2, where fp16 has three bits
// more than bf16 at the same rate.  Two things would still lose digits.  (1) A singular value far below the others grows by a = 3.44
// a step, 485 times in five, and so does a rounding of X in its direction.  X is therefore kept as the sum of two fp16
// numbers (22 bits); the products take the upper one, a X both.  (2) The terms of B X cancel those of a X where a
// singular value is near 1, and most of them is the diagonal of B.  The diagonals of A and B are kept apart in fp32, and the
// fp16 matrices have zeros there:
//   B_ij = b A_ij + c ((A'A')_ij + (alpha_i + alpha_j) A_ij),  beta_i = b alpha_i + c ((A'A')_ii + alpha_i^2),
//   X_i  = (a + beta_i) X_i + (B' X)_i                      (A' = A without its diagonal alpha, B' likewise)
// and alpha_i is the sum of squares of a row of X in full, not of its upper half: an identity, whose roundings all
// align, is served to 1e-6 (4e-3 with the product's diagonal).  Five steps, relative to 64 bits: 5e-4 to 8e-4 for full spectra, 1e-3
// for a matrix of rank 32, 2e-3 for rank one, where a plain bf16 iteration is off by 1e-2, 0.2 and 1.
//
// Range.  X is held times a power of two (scale_of): 256 at the start, where its elements are near 1/sqrt(m n), and 1 from the first step
// on.  Where G is smaller than eps, d = |G|_F / eps times, X stays small until the steps have grown it, each by a at most: there it is
// held at 64 to 256 times the bound d a^k of its norm, so that it keeps its 22 bits however small d is.
//
// Layout.  X, A and B live in the workspace as blocks of 64x64 fp16 (8 KB), in the 128-byte swizzle that the tensor core
// wants, the row blocks of a column block one after the other.  A tile of 128 rows by 64 columns is then 16 KB in a row, one
// copy, K-major; and the same blocks serve as the MN-major operand of B X, whose reduction runs over the rows of X.
// The blocks are padded with zeros, so ragged sizes need no special code.
//
// A and B are symmetric: only tiles on or below the diagonal are computed, and written twice.
//
// One launch per product, for up to 32 matrices at once (their tiles in one list), in one of two kernels:
//   ns_pair_kernel   256x256 tiles, each by a pair of blocks (cta_group::2), persistent: large products.  What bounds it is the
//                    feed from L2, about 57 bytes a cycle and SM: a single block's 128x256 tile needs 94 at the rate
//                    of the tensor core and took 850 cycles for a reduction of 64, a pair needs 64.
//   ns_tile_kernel   a 128x128 tile a block, two blocks on an SM: small products; the reduction of a symmetric
//                    one may be split over up to four blocks of a cluster, whose sums meet through distributed shared memory.
// The epilogues are the same: a warp has 32 rows by 64 columns in shared memory in fp32, walks them four rows at a time, so
// that what it reads and writes in the blocks is 512 bytes in a row, and writes the mirror image from the transposed reads.
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstring>

#include <cuda_fp16.h>

#include "orthogonalize.cuh"
#include "tc_ptx.cuh"
#include "tconv_host.cuh"

namespace {

constexpr float kA = twn_detail::kNsA, kB = twn_detail::kNsB, kC = twn_detail::kNsC;
constexpr float kStart = 256.0f;             // X of the first step is this much larger
constexpr int kMaxItems = twn_detail::kNsMaxItems;
constexpr int kBlockBytes = 8192, kBlockHalves = kBlockBytes / 2;
constexpr int kOpBytes = 2 * kBlockBytes, kStageBytes = 2 * kOpBytes;     // 128 rows (or columns) of each operand by 64
constexpr int kPairStages = 5;
constexpr int kEpiWarps = 8, kWarpTile = 32 * 64;
constexpr int kNsThreads = 32 * (2 + kEpiWarps);
constexpr int kMaxSplit = 4;                 // blocks that share a tile's reduction: a cluster
constexpr int kMaxParts = 512;               // of a matrix's sum of squares
constexpr long long kPartElements = 8192;
constexpr int kSweepBlock = 256;
constexpr int kMaxSteps = 32;
constexpr size_t kScaleBytes = 8 * kMaxSteps;

enum { kGram = 0, kSquare = 1, kApply = 2 };

struct NsItem {
    const void *G;               // the update; NULL for Muon, whose update is
    const float *dW;             //   V, or dW + momentum V (look ahead), with
    float *V;                    //   V = momentum V + dW, which the first sweep writes
    void *O;
    uint16_t *x[2], *lo, *A, *B; // blocks
    float *alpha, *beta;         // diagonals
    float2 *scale;               // what the sums of a step's A, and of its B X, are multiplied by
    float *squares;              // [cb][64 rb]: sums of squares of 64 elements of a row of X
    double *part;                // sums of squares
    long long count;             // elements
    int m, n, rb, cb;            // shorter and longer side; row and column blocks of X
    int parts;
    int first;                   // its first unit in the list of the launch
    int split;                   // blocks that share a reduction of the launch
    float out_scale;
    uint8_t g_bf16, o_bf16, tall, vec_in, vec_out, sym_pair, apply_pair;
};

struct NsParams {
    NsItem item[kMaxItems];
    int count, units, step, last, steps;
    float momentum, eps;
    int look_ahead;
    int32_t *status;
    const uint16_t *base;        // of the blocks: rows of the tensor maps count from here
};

__device__ __forceinline__ int item_of(const NsParams &P, int unit)
{
    int t = 0;
    while (t + 1 < P.count && unit >= P.item[t + 1].first) ++t;
    return t;
}

// Block (R, C) of a matrix of rb row blocks.
__device__ __forceinline__ size_t block_at(int R, int C, int rb) { return ((size_t)C * rb + R) * kBlockHalves; }
// Element (r, c) of a block: rows of 128 bytes, their 16-byte pieces exchanged by the row's number modulo 8.
__device__ __forceinline__ int in_block(int r, int c) { return r * 64 + ((((c >> 3) ^ r) & 7) << 3) + (c & 7); }
// Eight elements of row r of the whole matrix from column c on (a multiple of 8).
__device__ __forceinline__ size_t piece_at(int r, int c, int rb) { return block_at(r >> 6, c >> 6, rb) + in_block(r & 63, c & 63); }

__device__ __forceinline__ float muon_update(const NsParams &P, float v, float d)
{
    return P.look_ahead ? __fadd_rn(d, __fmul_rn(P.momentum, v)) : v;
}
__device__ __forceinline__ float element(const NsItem &it, const NsParams &P, long long i)
{
    if (it.V) return muon_update(P, it.V[i], it.dW[i]);
    return it.g_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(it.G)[i]) : static_cast<const float *>(it.G)[i];
}

// Sum over a block of kSweepBlock threads, in a fixed order, in every thread.
__device__ __forceinline__ double block_sum(double s, double *red)
{
    for (int o = 16; o > 0; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    s = red[0];
    for (int w = 1; w < kSweepBlock / 32; ++w) s += red[w];
    return s;
}

// Eight elements from i on, a multiple of 8 in an aligned tensor; for Muon's first sweep with the momentum updated.
template <bool UPDATE> __device__ __forceinline__ void elements8(const NsItem &it, const NsParams &P, long long i, float (&g)[8])
{
    if (it.V) {
        float4 *v4 = reinterpret_cast<float4 *>(it.V + i);
        const float4 *d4 = reinterpret_cast<const float4 *>(it.dW + i);
        float4 v[2] = {v4[0], v4[1]};
        const float4 d[2] = {d4[0], d4[1]};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float *const vp = &v[h].x;
            const float *const dp = &d[h].x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (UPDATE) vp[j] = __fadd_rn(__fmul_rn(P.momentum, vp[j]), dp[j]);
                g[4 * h + j] = muon_update(P, vp[j], dp[j]);
            }
            if (UPDATE) v4[h] = v[h];
        }
    } else if (it.g_bf16) {
        const uint4 w = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(it.G) + i);
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { g[2 * j] = __uint_as_float(ws[j] << 16); g[2 * j + 1] = __uint_as_float(ws[j] & 0xFFFF0000u); }
    } else {
        const float4 *g4 = reinterpret_cast<const float4 *>(static_cast<const float *>(it.G) + i);
        const float4 a = g4[0], b = g4[1];
        g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w; g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
    }
}

// Sum of squares of every matrix, in fp64 and in a fixed order; for Muon the momentum is updated on the way.
__global__ void __launch_bounds__(kSweepBlock) ns_norm_kernel(const __grid_constant__ NsParams P)
{
    __shared__ double red[kSweepBlock / 32];
    pdl_begin();
    for (int u = blockIdx.x; u < P.units; u += gridDim.x) {
        const NsItem &it = P.item[item_of(P, u)];
        const int part = u - it.first;
        const long long per = ((it.count + it.parts - 1) / it.parts + 2047) / 2048 * 2048;
        const long long begin = min(it.count, part * per), end = min(it.count, begin + per);
        const long long whole = it.vec_in ? begin + (end - begin) / 8 * 8 : begin;
        double s0 = 0.0, s1 = 0.0;
#pragma unroll 2
        for (long long i = begin + 8 * threadIdx.x; i < whole; i += 8 * kSweepBlock) {
            float g[8];
            elements8<true>(it, P, i, g);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                s0 += (double)g[j] * (double)g[j];
                s1 += (double)g[j + 1] * (double)g[j + 1];
            }
        }
        for (long long i = whole + threadIdx.x; i < end; i += kSweepBlock) {
            double g;
            if (it.V) {
                const float d = it.dW[i], v = __fadd_rn(__fmul_rn(P.momentum, it.V[i]), d);
                it.V[i] = v;
                g = muon_update(P, v, d);
            } else {
                g = element(it, P, i);
            }
            s0 += g * g;
        }
        const double s = block_sum(s0 + s1, red);
        if (threadIdx.x == 0) it.part[part] = s;
    }
}

// Eight values as two fp16 numbers each: the upper halves in one 16-byte piece, what they leave in another.
__device__ __forceinline__ uint32_t half2_bits(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 half2_of(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ uint4 pack_half8(const float (&f)[8])
{
    return make_uint4(half2_bits(f[0], f[1]), half2_bits(f[2], f[3]), half2_bits(f[4], f[5]), half2_bits(f[6], f[7]));
}
__device__ __forceinline__ void unpack_half8(const uint4 &w, float (&f)[8])
{
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 v = half2_of(ws[j]);
        f[2 * j] = v.x;
        f[2 * j + 1] = v.y;
    }
}
__device__ __forceinline__ uint4 pack_rest8(const float (&f)[8], const uint4 &hi)
{
    float h[8], l[8];
    unpack_half8(hi, h);
#pragma unroll
    for (int j = 0; j < 8; ++j) l[j] = f[j] - h[j];
    return pack_half8(l);
}
// The sum of squares of a row's 64 elements in a block, from the eight lanes that have them, in lanes 0, 8, 16, 24.
__device__ __forceinline__ float row_squares(const float (&f)[8])
{
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) q = fmaf(f[j], f[j], q);
    for (int o = 1; o < 8; o <<= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
    return q;
}

// The power of two that the X before a step is held times, for |G|_F / eps = d below 1 and 1 at eps or above: see the top.
__device__ __forceinline__ float scale_of(double d, int step, int steps)
{
    if (step == steps) return 1.0f;
    if (d >= 1.0) return step == 0 ? kStart : 1.0f;
    for (int k = 0; k < step; ++k) d *= (double)kA;
    return d > 0.0 ? (float)ldexp(1.0, min(126, max(0, 7 - ilogb(d)))) : 1.0f;
}

// X of the first step, a block of 64x64 at a time: normalised, split into two fp16 numbers, padded with zeros.
__global__ void __launch_bounds__(kSweepBlock) ns_start_kernel(const __grid_constant__ NsParams P)
{
    __shared__ double red[kSweepBlock / 32];
    __shared__ float tile[64][65];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int have = -1;
    float pre = 1.0f, factor = 0.0f, nan = 0.0f;
    pdl_begin();
    for (int u = blockIdx.x; u < P.units; u += gridDim.x) {
        const int t = item_of(P, u);
        const NsItem &it = P.item[t];
        const int b = u - it.first, R = b % it.rb, C = b / it.rb;
        if (t != have) {
            double s = 0.0;
            for (int p = threadIdx.x; p < it.parts; p += kSweepBlock) s += it.part[p];
            const double norm = sqrt(block_sum(s, red));
            if (b == 0 && threadIdx.x == 0 && P.status && !isfinite(norm)) atomicMin(P.status, (int)TWN_ERR_NONFINITE);
            const double d = norm < (double)P.eps ? norm / (double)P.eps : 1.0;
            if (b == 0 && threadIdx.x < P.steps) {
                const float inverse = 1.0f / scale_of(d, threadIdx.x, P.steps);
                it.scale[threadIdx.x] = make_float2(inverse * inverse, inverse * scale_of(d, threadIdx.x + 1, P.steps));
            }
            // in two factors, so that neither leaves the range of fp32
            pre = norm > 1e18 ? 0x1p-100f : norm < 1e-18 ? 0x1p100f : 1.0f;
            factor = norm == 0.0 ? 0.0f : (float)((double)scale_of(d, 0, P.steps) / (fmax(norm, (double)P.eps) * (double)pre));
            nan = norm == norm ? 0.0f : __uint_as_float(0x7FC00000u);      // fmax drops a NaN
            have = t;
        }
        const int r0 = 64 * R, c0 = 64 * C;
        const bool direct = it.vec_in && !it.tall && it.n % 8 == 0;
        if (!direct) {
            // rows of G along the threads of a warp
            __syncthreads();
            const int rows = it.tall ? it.n : it.m, cols = it.tall ? it.m : it.n;
            const int j = threadIdx.x & 63, i0 = threadIdx.x >> 6, col = (it.tall ? r0 : c0) + j, row = (it.tall ? c0 : r0) + i0;
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = row + 4 * k < rows && col < cols ? element(it, P, (long long)(row + 4 * k) * cols + col) : 0.0f;
            if (it.tall) {
#pragma unroll
                for (int k = 0; k < 16; ++k) tile[j][i0 + 4 * k] = v[k];
            } else {
#pragma unroll
                for (int k = 0; k < 16; ++k) tile[i0 + 4 * k][j] = v[k];
            }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int rr = 8 * warp + 4 * k + (lane >> 3), cc = 8 * (lane & 7), r = r0 + rr, c = c0 + cc;
            const bool in = r < it.m && c < it.n;
            float f[8];
            if (direct) {
                if (in) elements8<false>(it, P, (long long)r * it.n + c, f);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = tile[rr][cc + j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = in && c + j < it.n ? f[j] * pre * factor + nan : 0.0f;
            const size_t at = block_at(R, C, it.rb) + in_block(rr, cc);
            const uint4 hi = pack_half8(f);
            *reinterpret_cast<uint4 *>(it.x[0] + at) = hi;
            *reinterpret_cast<uint4 *>(it.lo + at) = pack_rest8(f, hi);
            const float q = row_squares(f);
            if ((lane & 7) == 0) it.squares[(size_t)C * (64 * it.rb) + r] = q;
        }
    }
}

// ---- PTX of the products ---------------------------------------------------------------------------------------------------
// Rows of 128 bytes from row `row` of a matrix of blocks on, by either block of a pair; the barrier is at this address in the
// first of them.
__device__ __forceinline__ void pair_load(void *dst, const CUtensorMap *map, uint32_t bar, int row)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(row) : "memory");
}
// D[tmem] (+)= A[smem] B[smem]^T, fp16, issued by the calling thread alone; PAIR: by that of the first block for both.
template <bool PAIR> __device__ __forceinline__ void ns_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc)
{
    if (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
// The barrier at this address in both blocks gets one arrival when the MMAs so far are done.
__device__ __forceinline__ void pair_commit(void *bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ uint32_t of_block(uint32_t addr, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ float4 ld_block(uint32_t cluster_addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
// Without waiting for what this block has written.
__device__ __forceinline__ void cluster_done()
{
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}

// ---- epilogue ----------------------------------------------------------------------------------------------------------------
// A warp's 32 x 64 sums in shared memory: 16-byte piece 2 p + h of row r lies where a warp's row-wise writes, reads of four
// rows by eight pieces of like h, and reads of eight columns by four runs of eight rows are all free of bank conflicts.
__device__ __forceinline__ int slot_of(int r, int p, int h) { return r * 64 + h * 32 + (((p ^ r ^ (r >> 3) ^ (h << 2)) & 7) << 2); }

// 64 columns of the accumulator of a warp's 32 rows.
__device__ __forceinline__ void dump_sums(uint32_t taddr, float *buf)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        uint32_t v[32];
        tmem_ld32(taddr + 32 * g, v);
        tmem_wait_ld(v);
#pragma unroll
        for (int p = 0; p < 8; ++p)
            *reinterpret_cast<uint4 *>(buf + slot_of(lane, 4 * g + (p >> 1), p & 1)) = make_uint4(v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]);
    }
}

__device__ __forceinline__ void row_sums8(const float *buf, int r, int p, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(buf + slot_of(r, p, 0)), b = *reinterpret_cast<const float4 *>(buf + slot_of(r, p, 1));
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void column_sums8(const float *buf, int r, int c, float (&v)[8])      // rows r .. r + 7
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = buf[slot_of(r + e, c >> 3, (c >> 2) & 1) + (c & 3)];
}
__device__ __forceinline__ void load8(const float *p, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// The diagonal of A for a warp's rows, if its tile lies on it: the sums of squares of whole rows of X, 512 blocks of columns at a time, and
// those sums.  It needs no product, so it is done while they run.
__device__ __forceinline__ void write_alpha(const NsItem &it, float unscale, int r0, int c0)
{
    if (r0 < c0 || r0 >= c0 + 64) return;
    const int r = r0 + (threadIdx.x & 31);
    float a = 0.0f;
#pragma unroll 1
    for (int g0 = 0; g0 < it.cb; g0 += 512) {
        float run = 0.0f;
        const int end = min(g0 + 512, it.cb);
#pragma unroll 16
        for (int g = g0; g < end; ++g) run += it.squares[(size_t)g * (64 * it.rb) + r];
        a += run;
    }
    it.alpha[r] = a * unscale;
}
__device__ __forceinline__ float of_square(float sum, float a, float alphas) { return kB * a + kC * (sum + alphas * a); }
__device__ __forceinline__ float of_diagonal(float sum, float alpha) { return kB * alpha + kC * (sum + alpha * alpha); }

// Where a lane's pieces of a warp's tile lie: unit u has row r0 + 4 u + lane / 8, piece lane % 8 (an odd unit's row has the other
// bit 2, which the swizzle exchanges); of the mirror image row c0 + 8 u + lane / 4, piece lane % 4 of the warp's four.
struct Pieces {
    size_t even;
    __device__ __forceinline__ Pieces(const NsItem &it, int r0, int c0)
    {
        const int lane = threadIdx.x & 31;
        even = block_at(r0 >> 6, c0 >> 6, it.rb) + in_block((r0 & 63) + (lane >> 3), 8 * (lane & 7));
    }
    __device__ __forceinline__ size_t operator()(int u) const { return (u & 1 ? even ^ 32 : even) + 256 * u; }
};
__device__ __forceinline__ size_t mirror_piece(const NsItem &it, int r0, int c0)
{
    const int lane = threadIdx.x & 31;
    return block_at(c0 >> 6, r0 >> 6, it.rb) + in_block(lane >> 2, (r0 & 63) + 8 * (lane & 3));
}

// What a warp's tile of rows r0 .. r0 + 31 and columns c0 .. c0 + 63 reads from global memory, eight units of four rows: loaded
// before the sums are there.
template <int PHASE> struct Ahead;
template <> struct Ahead<kGram> {
    float unscale;
    __device__ __forceinline__ void load(const NsItem &it, const NsParams &P, int, int) { unscale = it.scale[P.step].x; }
};
template <> struct Ahead<kSquare> {
    uint4 a[8];
    float row[8], column[8];
    __device__ __forceinline__ void load(const NsItem &it, const NsParams &, int r0, int c0)
    {
        const int lane = threadIdx.x & 31;
        const uint16_t *const A = it.A;
        const float *const alpha = it.alpha + r0 + (lane >> 3);
        const Pieces at(it, r0, c0);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            a[u] = *reinterpret_cast<const uint4 *>(A + at(u));
            row[u] = alpha[4 * u];
        }
        load8(it.alpha + c0 + 8 * (lane & 7), column);
    }
};
template <> struct Ahead<kApply> {
    uint4 hi[4], lo[4];          // of the first four units
    float row[8], unscale;
    __device__ __forceinline__ void load4(const NsItem &it, const NsParams &P, int r0, int c0, int u0)
    {
        const uint16_t *const x = it.x[P.step & 1], *const rest = it.lo;
        const Pieces at(it, r0, c0);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            hi[u] = *reinterpret_cast<const uint4 *>(x + at(u0 + u));
            lo[u] = *reinterpret_cast<const uint4 *>(rest + at(u0 + u));
        }
    }
    __device__ __forceinline__ void load(const NsItem &it, const NsParams &P, int r0, int c0)
    {
        load4(it, P, r0, c0, 0);
        unscale = it.scale[P.step].y;
#pragma unroll
        for (int u = 0; u < 8; ++u) row[u] = (it.beta + r0 + ((threadIdx.x & 31) >> 3))[4 * u];
    }
};

// Symmetric products: a warp's tile and its mirror image.
template <int PHASE>
__device__ __forceinline__ void finish_symmetric(const NsItem &it, const NsParams &P, const Ahead<PHASE> &ahead, const float *buf, int r0, int c0, bool mirror)
{
    const int lane = threadIdx.x & 31;
    const bool diagonal = r0 >= c0 && r0 < c0 + 64;
    float unscale = 1.0f;
    if constexpr (PHASE == kGram) unscale = ahead.unscale;
    uint16_t *const to = PHASE == kGram ? it.A : it.B;
    const int p = lane & 7;
    const Pieces at(it, r0, c0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int r = 4 * u + (lane >> 3);
        float v[8];
        row_sums8(buf, r, p, v);
        if constexpr (PHASE == kSquare) {
            float a[8];
            unpack_half8(ahead.a[u], a);
            if (diagonal)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c0 + 8 * p + j == r0 + r) it.beta[r0 + r] = of_diagonal(v[j], ahead.row[u]);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = of_square(v[j], a[j], ahead.row[u] + ahead.column[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= unscale;
        }
        if (diagonal)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + 8 * p + j == r0 + r) v[j] = 0.0f;
        *reinterpret_cast<uint4 *>(to + at(u)) = pack_half8(v);
    }
    if (!mirror) return;
    const int r = 8 * (lane & 3);
    const size_t mirrored = mirror_piece(it, r0, c0);
    float alpha_r[8];
    if (PHASE == kSquare) load8(it.alpha + r0 + r, alpha_r);
#pragma unroll 4
    for (int u = 0; u < 8; ++u) {
        const int c = 8 * u + (lane >> 2);
        const size_t at = mirrored + 512 * u;
        float v[8];
        column_sums8(buf, r, c, v);
        if constexpr (PHASE == kSquare) {
            float a[8];
            unpack_half8(*reinterpret_cast<const uint4 *>(it.A + at), a);
            const float alpha_c = it.alpha[c0 + c];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = of_square(v[j], a[j], alpha_r[j] + alpha_c);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= unscale;
        }
        *reinterpret_cast<uint4 *>(to + at) = pack_half8(v);
    }
}

// The same where `split` blocks of a cluster, from rank `first` on, hold a part of the sums each at this address.  Of the four runs of
// eight rows of a warp's tile a block takes those that are `me` modulo `split`: it reads all parts at once, 128 bytes in a row at a time
// (a row a thread, 16 bytes each from another one, took 7 to 12 us for four blocks), adds them in the blocks' order, and leaves the
// sum in its own part, which nobody else reads there, for the mirror image.
template <int PHASE>
__device__ __forceinline__ void finish_split(const NsItem &it, const NsParams &P, float *buf, uint32_t first, float unscale, int r0, int c0, bool mirror, int me, int split)
{
    const int lane = threadIdx.x & 31, p = lane & 7;
    const bool diagonal = r0 >= c0 && r0 < c0 + 64;
    uint16_t *const to = PHASE == kGram ? it.A : it.B;
    const uint32_t addr = smem_u32(buf);
    const Pieces at(it, r0, c0);
    float alpha_c[8];
    if (PHASE == kSquare) load8(it.alpha + c0 + 8 * p, alpha_c);
#pragma unroll 1
    for (int k = me; k < 4; k += split) {
        float4 part[kMaxSplit][4];
        uint4 aw[2];
        float alpha[2] = {0.0f, 0.0f};
#pragma unroll
        for (int g = 0; g < kMaxSplit; ++g) {
            if (g >= split) break;
            const uint32_t from = of_block(addr, first + g);
#pragma unroll
            for (int h = 0; h < 4; ++h) part[g][h] = ld_block(from + 4 * slot_of(8 * k + 4 * (h >> 1) + (lane >> 3), p, h & 1));
        }
        if (PHASE == kSquare)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                aw[h] = *reinterpret_cast<const uint4 *>(it.A + at(2 * k + h));
                alpha[h] = it.alpha[r0 + 8 * k + 4 * h + (lane >> 3)];
            }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 8 * k + 4 * h + (lane >> 3);
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (&part[0][2 * h + (j >> 2)].x)[j & 3];
#pragma unroll
            for (int g = 1; g < kMaxSplit; ++g) {
                if (g >= split) break;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += (&part[g][2 * h + (j >> 2)].x)[j & 3];
            }
            if (PHASE == kSquare) {
                float a[8];
                unpack_half8(aw[h], a);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (diagonal && c0 + 8 * p + j == r0 + r) it.beta[r0 + r] = of_diagonal(v[j], alpha[h]);
                    v[j] = of_square(v[j], a[j], alpha[h] + alpha_c[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= unscale;
            }
            if (diagonal)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c0 + 8 * p + j == r0 + r) v[j] = 0.0f;
            *reinterpret_cast<uint4 *>(to + at(2 * k + h)) = pack_half8(v);
            if (mirror) {
                *reinterpret_cast<float4 *>(buf + slot_of(r, p, 0)) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4 *>(buf + slot_of(r, p, 1)) = make_float4(v[4], v[5], v[6], v[7]);
            }
        }
        if (mirror) {
            __syncwarp();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = 32 * h + lane;
                float v[8];
                column_sums8(buf, 8 * k, c, v);
                *reinterpret_cast<uint4 *>(to + piece_at(c0 + c, r0 + 8 * k, it.rb)) = pack_half8(v);
            }
        }
    }
}

__device__ __forceinline__ void store_out(const NsItem &it, long long at, float v)
{
    if (it.o_bf16) static_cast<__nv_bfloat16 *>(it.O)[at] = __float2bfloat16_rn(v);
    else static_cast<float *>(it.O)[at] = v;
}
__device__ __forceinline__ void store_out8(const NsItem &it, long long at, const float (&v)[8])
{
    if (it.o_bf16) {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(it.O) + at) =
            make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    } else {
        float4 *o = reinterpret_cast<float4 *>(static_cast<float *>(it.O) + at);
        o[0] = make_float4(v[0], v[1], v[2], v[3]);
        o[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// X of the next step, or the result.  DEEP: the second half of the operands is on its way while the first is worked on (32 registers).
template <bool DEEP> __device__ __forceinline__ void finish_apply(const NsItem &it, const NsParams &P, Ahead<kApply> &ahead, float *buf, int r0, int c0)
{
    const int lane = threadIdx.x & 31, p = lane & 7, cur = P.step & 1;
    const float unscale = ahead.unscale;
    uint16_t *const next = it.x[cur ^ 1], *const rest = it.lo;
    const Pieces at(it, r0, c0);
    Ahead<kApply> second;
    if (DEEP) second.load4(it, P, r0, c0, 4);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        if (!DEEP && u == 4) ahead.load4(it, P, r0, c0, 4);
        const Ahead<kApply> &now = DEEP && u >= 4 ? second : ahead;
        const int r = 4 * u + (lane >> 3);
        const float k = kA + ahead.row[u];
        float v[8], h[8], l[8];
        row_sums8(buf, r, p, v);
        unpack_half8(now.hi[u & 3], h);
        unpack_half8(now.lo[u & 3], l);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (k * (h[j] + l[j]) + v[j]) * unscale;
        if (P.last) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= it.out_scale;
            if (it.vec_out && !it.tall) {
                if (r0 + r < it.m && c0 + 8 * p < it.n) store_out8(it, (long long)(r0 + r) * it.n + c0 + 8 * p, v);
            } else {
                *reinterpret_cast<float4 *>(buf + slot_of(r, p, 0)) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4 *>(buf + slot_of(r, p, 1)) = make_float4(v[4], v[5], v[6], v[7]);
            }
        } else {
            const uint4 h2 = pack_half8(v);
            *reinterpret_cast<uint4 *>(next + at(u)) = h2;
            *reinterpret_cast<uint4 *>(rest + at(u)) = pack_rest8(v, h2);
            const float q = row_squares(v);
            if (p == 0) it.squares[(size_t)(c0 >> 6) * (64 * it.rb) + r0 + r] = q;
        }
    }
    if (!P.last || (it.vec_out && !it.tall)) return;
    __syncwarp();
    if (it.tall && it.vec_out) {
#pragma unroll 2
        for (int u = 0; u < 8; ++u) {
            const int c = 8 * u + (lane >> 2), r = 8 * (lane & 3);
            float v[8];
            column_sums8(buf, r, c, v);
            if (c0 + c < it.n && r0 + r < it.m) store_out8(it, (long long)(c0 + c) * it.m + r0 + r, v);
        }
    } else if (it.tall) {
        if (r0 + lane < it.m)
            for (int c = 0; c < 64 && c0 + c < it.n; ++c)
                store_out(it, (long long)(c0 + c) * it.m + r0 + lane, buf[slot_of(lane, c >> 3, (c >> 2) & 1) + (c & 3)]);
    } else {
        for (int r = 0; r < 32 && r0 + r < it.m; ++r)
            for (int c = lane; c < 64 && c0 + c < it.n; c += 32)
                store_out(it, (long long)(r0 + r) * it.n + c0 + c, buf[slot_of(r, c >> 3, (c >> 2) & 1) + (c & 3)]);
    }
}

// Row `u` of a triangle that is written row by row, and what is left of u in it.
__device__ __forceinline__ int triangle_row(int u, int *column)
{
    int i = (int)((sqrtf(8.0f * (float)u + 1.0f) - 1.0f) * 0.5f);
    while (i * (i + 1) / 2 > u) --i;
    while ((i + 1) * (i + 2) / 2 <= u) ++i;
    *column = u - i * (i + 1) / 2;
    return i;
}

template <int PHASE> __device__ __forceinline__ int reduction_blocks(const NsItem &it) { return PHASE == kGram ? (it.n + 63) >> 6 : (it.m + 63) >> 6; }

// fp16 operands, fp32 accumulator; B MN-major where it is X
template <int PHASE> __host__ __device__ constexpr uint32_t ns_idesc(int M, int N)
{
    return (1u << 4) | (PHASE == kApply ? 1u << 16 : 0u) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// One reduction block: four MMAs of 16.
template <int PHASE, bool PAIR> __device__ __forceinline__ void ns_mma_block(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool first)
{
    constexpr uint64_t kStep = PHASE == kApply ? (16 * 128) >> 4 : 32 >> 4;      // 16 rows of the reduction, or 16 columns
    ns_mma<PAIR>(d, a, b, idesc, first ? 0u : 1u);
    ns_mma<PAIR>(d, a + 2, b + kStep, idesc, 1u);
    ns_mma<PAIR>(d, a + 4, b + 2 * kStep, idesc, 1u);
    ns_mma<PAIR>(d, a + 6, b + 3 * kStep, idesc, 1u);
}

// ---- large products ------------------------------------------------------------------------------------------------------
// 256x256 tiles by pairs of blocks: a block has 128 rows of A and 128 of B's 256 columns in shared memory and 128 rows by 256
// columns of the result in tensor memory, twice, so the epilogue of a tile runs beside the next one.  Both blocks' copies count on the
// barrier of the first, whose thread issues the MMAs for both.
struct __align__(1024) PairSmem {
    uint8_t ring[kPairStages][kStageBytes];
    float sums[kEpiWarps][kWarpTile];
    unsigned long long full[kPairStages], empty[kPairStages], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    volatile int abort_flag;
};

template <int PHASE>
__global__ void __launch_bounds__(kNsThreads, 1)
ns_pair_kernel(const __grid_constant__ CUtensorMap rows128, const __grid_constant__ CUtensorMap rows64, const __grid_constant__ NsParams P)
{
    if (gridDim.x <= kPdlBlocks) pdl_launch_dependents();
    extern __shared__ uint8_t smem_raw[];
    PairSmem *sm = reinterpret_cast<PairSmem *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    volatile int *abort_flag = &sm->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();

    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; ++s) { mbar_init(&sm->full[s], 1); mbar_init(&sm->empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&sm->acc_full[s], 1); mbar_init(&sm->acc_empty[s], 2 * kEpiWarps); }
        sm->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm->tmem_base)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    pdl_wait();
    const uint32_t tmem = sm->tmem_base;
    const int cur = P.step & 1;
    const int pairs = gridDim.x >> 1, pair = blockIdx.x >> 1;

    // tile (I, J) of unit u
    auto tile_of = [&](const NsItem &it, int u, int &I, int &J) {
        u -= it.first;
        if (PHASE == kApply) {
            const int rows = it.rb >> 2;
            I = u % rows;
            J = u / rows;
        } else {
            I = triangle_row(u, &J);
        }
    };

    if (warp == 0) {
        if (elect_one()) {
            uint32_t s = 0, ph = 0;
            bool ok = true;
            for (int u = pair; u < P.units && ok; u += pairs) {
                const NsItem &it = P.item[item_of(P, u)];
                int I, J;
                tile_of(it, u, I, J);
                const uint16_t *const src_a = PHASE == kGram ? it.x[cur] : PHASE == kSquare ? it.A : it.B;
                const uint16_t *const src_b = PHASE == kSquare ? it.A : it.x[cur];
                // rows of 128 bytes from the first of the workspace's blocks on
                const int a_row = (int)((src_a - P.base) >> 6), b_row = (int)((src_b - P.base) >> 6);
                const int kb = reduction_blocks<PHASE>(it);
                // a tile on the diagonal has the same rows on both sides, in both blocks
                const bool same = PHASE != kApply && I == J;
                for (int k = 0; k < kb; ++k) {
                    uint8_t *const st = sm->ring[s];
                    if (!mbar_wait(&sm->empty[s], ph ^ 1u, abort_flag, P.status, 20)) { ok = false; break; }
                    if (rank == 0) mbar_expect_tx(&sm->full[s], same ? 2 * kOpBytes : 2 * kStageBytes);
                    const uint32_t bar = of_block(smem_u32(&sm->full[s]), 0);
                    pair_load(st, &rows128, bar, a_row + 64 * (k * it.rb + 4 * I + 2 * (int)rank));
                    if (PHASE == kApply) {
                        for (int j = 0; j < 2; ++j)
                            pair_load(st + kOpBytes + j * kBlockBytes, &rows64, bar, b_row + 64 * ((4 * J + 2 * (int)rank + j) * it.rb + k));
                    } else if (!same) {
                        pair_load(st + kOpBytes, &rows128, bar, b_row + 64 * (k * it.rb + 4 * J + 2 * (int)rank));
                    }
                    if (++s == kPairStages) { s = 0; ph ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            uint32_t s = 0, ph = 0, lu = 0;
            bool ok = true;
            const uint32_t ring = smem_u32(sm->ring);
            const uint64_t a0 = smem_desc_sw128(ring);
            const uint64_t b0 = PHASE == kApply ? smem_desc_mn_sw128(ring + kOpBytes, kBlockBytes) : smem_desc_sw128(ring + kOpBytes);
            constexpr uint32_t idesc = ns_idesc<PHASE>(256, 256);
            for (int u = pair; u < P.units && ok; u += pairs, ++lu) {
                const NsItem &it = P.item[item_of(P, u)];
                int I, J;
                tile_of(it, u, I, J);
                const int kb = reduction_blocks<PHASE>(it);
                const uint64_t bt = PHASE != kApply && I == J ? a0 : b0;
                if (!mbar_wait(&sm->acc_empty[lu & 1], ((lu >> 1) & 1u) ^ 1u, abort_flag, P.status, 0)) break;
                tc_fence_after();
                for (int k = 0; k < kb; ++k) {
                    if (!mbar_wait(&sm->full[s], ph, abort_flag, P.status, 0)) { ok = false; break; }
                    tc_fence_after();
                    const uint64_t off = s * (uint64_t)(kStageBytes >> 4);
                    ns_mma_block<PHASE, true>(tmem + (lu & 1) * 256, a0 + off, bt + off, idesc, k == 0);
                    pair_commit(&sm->empty[s]);
                    if (++s == kPairStages) { s = 0; ph ^= 1u; }
                }
                if (ok) pair_commit(&sm->acc_full[lu & 1]);
            }
        }
    } else {
        const int q = warp & 3, set = (warp - 2) >> 2;
        float *const buf = sm->sums[warp - 2];
        uint32_t lu = 0;
        for (int u = pair; u < P.units; u += pairs, ++lu) {
            const NsItem &it = P.item[item_of(P, u)];
            int I, J;
            tile_of(it, u, I, J);
            const int r0 = 256 * I + 128 * (int)rank + 32 * q;
            bool ok = true;
#pragma unroll 1
            for (int b = set; b < 4; b += 2) {
                const int c0 = 256 * J + 64 * b;
                Ahead<PHASE> ahead;
                ahead.load(it, P, r0, c0);
                if constexpr (PHASE == kGram) write_alpha(it, ahead.unscale, r0, c0);
                if (b < 2 && !mbar_wait_warp(&sm->acc_full[lu & 1], (lu >> 1) & 1u, abort_flag, P.status, 32)) { ok = false; break; }
                tc_fence_after();
                dump_sums(tmem + ((uint32_t)(32 * q) << 16) + (lu & 1) * 256 + 64 * b, buf);
                __syncwarp();
                if (b >= 2) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_at(of_block(smem_u32(&sm->acc_empty[lu & 1]), 0));
                }
                if constexpr (PHASE == kApply) finish_apply<true>(it, P, ahead, buf, r0, c0);
                else finish_symmetric<PHASE>(it, P, ahead, buf, r0, c0, J < I);
                __syncwarp();
            }
            if (!ok) break;
        }
    }

    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (sm->abort_flag) {
        // copies and products in flight end well within this
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
    }
    __syncthreads();
    cluster_sync();                                    // neither block's memory goes while the other may use it
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// ---- small products ------------------------------------------------------------------------------------------------------
// A 128x128 tile a block, two blocks on an SM with rings of three stages, or one with six where there are no more blocks than SMs (a
// block's reduction of 64 took 0.46 us with three, 1.5 times what the feed from L2 needs).  `split` blocks of a cluster share a tile's reduction; each leaves its sums in
// the shared memory that was its ring, and finishes every split-th unit of the whole tile.
//
// LONG: reductions of more than kChunk blocks.  The tensor core's sums are cut off at every addition (16 columns), half a unit in the last place too
// small on average; where the rows of X agree that goes all one way, 2^-25 of a sum for every 16 columns of a block's share (2 x 2^20 of
// mean 1: 7e-3 off in the result, 2 x 2^24: 8e-2).  So the sums of kChunk blocks, 2^-16 too small, are added in fp32 to those before, in
// tensor memory beside them, while the ring fills.
constexpr int kChunk = 128;
template <int STAGES> struct __align__(1024) TileSmem {
    union {
        uint8_t ring[STAGES][kStageBytes];
        float sums[kEpiWarps][kWarpTile];
    };
    unsigned long long full[STAGES], empty[STAGES], acc_full, acc_empty;
    uint32_t tmem_base;
    volatile int abort_flag;
};

// 64 columns of a warp's 32 rows: `more` added to `sums`, or put there.
__device__ __forceinline__ void add_sums(uint32_t sums, uint32_t more, bool first)
{
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        uint32_t v[32], w[32];
        tmem_ld32(more + 32 * g, v);
        tmem_wait_ld(v);
        if (!first) {
            tmem_ld32(sums + 32 * g, w);
            tmem_wait_ld(w);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(w[j]) + __uint_as_float(v[j]));
        }
        tmem_st32(sums + 32 * g, v);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
    }
}

template <int PHASE, int kTileStages, bool LONG>
__global__ void __launch_bounds__(kNsThreads, kTileStages > 3 ? 1 : 2) ns_tile_kernel(const __grid_constant__ NsParams P, bool clustered)
{
    pdl_launch_dependents();
    extern __shared__ uint8_t smem_raw[];
    using Smem = TileSmem<kTileStages>;
    Smem *sm = reinterpret_cast<Smem *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    volatile int *abort_flag = &sm->abort_flag;
    const int warp = threadIdx.x >> 5;
    constexpr uint32_t kColumns = LONG ? 256 : 128;      // of tensor memory

    if (threadIdx.x == 0) {
        for (int s = 0; s < kTileStages; ++s) { mbar_init(&sm->full[s], 1); mbar_init(&sm->empty[s], 1); }
        mbar_init(&sm->acc_full, 1);
        mbar_init(&sm->acc_empty, kEpiWarps);
        sm->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm->tmem_base)), "r"(kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // the tile's place needs the parameters alone: read while the kernel before this one ends
    const int cur = P.step & 1;
    const int u = blockIdx.x;
    const bool live = u < P.units;
    const NsItem &it = P.item[item_of(P, live ? u : 0)];
    const int split = PHASE == kApply ? 1 : it.split;
    int i = 0, j = 0, me = 0, k0 = 0, k1 = 0;
    if (live) {
        int t = u - it.first;
        if (PHASE == kApply) {
            const int rows = it.rb >> 1;
            i = t % rows;
            j = t / rows;
        } else {
            me = t & (split - 1);
            i = triangle_row(t / split, &j);
        }
        const int kb = reduction_blocks<PHASE>(it);
        k0 = (int)((long long)kb * me / split);        // a split leaves every block four reduction blocks or more
        k1 = (int)((long long)kb * (me + 1) / split);
    }
    const bool same = PHASE != kApply && i == j;       // the same rows on both sides
    const uint16_t *const src_a = PHASE == kGram ? it.x[cur] : PHASE == kSquare ? it.A : it.B;
    const uint16_t *const src_b = PHASE == kSquare ? it.A : it.x[cur];
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    const uint32_t tmem = sm->tmem_base;

    if (warp == 0) {
        if (elect_one()) {
            uint32_t s = 0, ph = 0;
            for (int k = k0; k < k1; ++k) {
                uint8_t *const st = sm->ring[s];
                if (!mbar_wait(&sm->empty[s], ph ^ 1u, abort_flag, P.status, 20)) break;
                mbar_expect_tx(&sm->full[s], same ? kOpBytes : kStageBytes);
                bulk_load(st, src_a + block_at(2 * i, k, it.rb), kOpBytes, &sm->full[s]);
                if (PHASE == kApply) {
                    for (int b = 0; b < 2; ++b)
                        bulk_load(st + kOpBytes + b * kBlockBytes, src_b + block_at(k, 2 * j + b, it.rb), kBlockBytes, &sm->full[s]);
                } else if (!same) {
                    bulk_load(st + kOpBytes, src_b + block_at(2 * j, k, it.rb), kOpBytes, &sm->full[s]);
                }
                if (++s == kTileStages) { s = 0; ph ^= 1u; }
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t ring = smem_u32(sm->ring);
            const uint64_t a0 = smem_desc_sw128(ring);
            const uint64_t b0 = same ? a0 : PHASE == kApply ? smem_desc_mn_sw128(ring + kOpBytes, kBlockBytes) : smem_desc_sw128(ring + kOpBytes);
            constexpr uint32_t idesc = ns_idesc<PHASE>(128, 128);
            uint32_t s = 0, ph = 0;
            bool ok = true;
            for (int k = k0; k < k1; ++k) {
                const int in_chunk = LONG ? (k - k0) % kChunk : k - k0;
                if (LONG && in_chunk == 0 && k > k0) {
                    tc_commit(&sm->acc_full);
                    if (!mbar_wait(&sm->acc_empty, ((k - k0) / kChunk - 1) & 1, abort_flag, P.status, 0)) { ok = false; break; }
                }
                if (!mbar_wait(&sm->full[s], ph, abort_flag, P.status, 0)) { ok = false; break; }
                tc_fence_after();
                const uint64_t off = s * (uint64_t)(kStageBytes >> 4);
                ns_mma_block<PHASE, false>(tmem, a0 + off, b0 + off, idesc, in_chunk == 0);
                tc_commit(&sm->empty[s]);
                if (++s == kTileStages) { s = 0; ph ^= 1u; }
            }
            if (ok) tc_commit(&sm->acc_full);
        }
    }
    __syncwarp();

    const int w = warp - 2, q = warp & 3, half = w >> 2;
    const int r0 = 128 * i + 32 * q, c0 = 128 * j + 64 * half;
    float unscale = 1.0f;
    if (warp >= 2 && live) {
        Ahead<PHASE> ahead;
        if (split == 1) ahead.load(it, P, r0, c0);
        if constexpr (PHASE == kGram) {
            unscale = it.scale[P.step].x;
            if (me == 0) write_alpha(it, unscale, r0, c0);
        }
        const uint32_t acc = tmem + ((uint32_t)(32 * q) << 16) + 64 * half;
        const int chunks = LONG ? (k1 - k0 + kChunk - 1) / kChunk : 1;
        bool ok = true;
        for (int c = 0; LONG && c + 1 < chunks && ok; ++c) {
            ok = mbar_wait_warp(&sm->acc_full, c & 1, abort_flag, P.status, 32);
            if (!ok) break;
            tc_fence_after();
            add_sums(acc + 128, acc, c == 0);
            tc_fence_before();
            __syncwarp();
            if ((threadIdx.x & 31) == 0) mbar_arrive(&sm->acc_empty);
        }
        // all products are done, so all copies have landed: the ring is free
        if (ok && mbar_wait_warp(&sm->acc_full, (chunks - 1) & 1, abort_flag, P.status, 32)) {
            tc_fence_after();
            if (LONG && chunks > 1) add_sums(acc + 128, acc, false);
            dump_sums(acc + (LONG && chunks > 1 ? 128 : 0), sm->sums[w]);
            tc_fence_before();
            __syncwarp();
            if (split == 1) {
                if constexpr (PHASE == kApply) finish_apply<(kTileStages > 3)>(it, P, ahead, sm->sums[w], r0, c0);
                else finish_symmetric<PHASE>(it, P, ahead, sm->sums[w], r0, c0, j < i);
            }
        }
    }
    __syncwarp();
    if constexpr (PHASE != kApply) {
        if (clustered) {
            cluster_sync();
            if (warp >= 2 && live && split > 1)
                finish_split<PHASE>(it, P, sm->sums[w], cluster_rank() & ~(uint32_t)(split - 1), unscale, r0, c0, j < i, me, split);
            __syncwarp();
            cluster_done();                            // no block's memory goes while another reads it
        }
    }

    tc_fence_before();
    __syncthreads();
    if (sm->abort_flag) {
        // copies and products in flight end well within this
        for (int k = 0; k < 64; ++k) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kColumns) : "memory");
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
size_t align256(size_t v) { return (v + 255) / 256 * 256; }

struct Shape {
    int64_t m, n, rb, cb, parts;
    bool fits, sym_pair, apply_pair;
};
constexpr int64_t kMaxShort = 32768, kMaxLong = 1 << 24, kPairLong = 1 << 17;
// How a matrix is served goes by its own sizes and by whether all matrices of the call are small (all_small), not by the others' sizes or
// number, so it has the same bits in every other batch.
Shape shape_of(int64_t rows, int64_t cols)
{
    Shape s = {};
    s.m = std::min(rows, cols);
    s.n = std::max(rows, cols);
    s.fits = s.m <= kMaxShort && s.n <= kMaxLong;
    if (!s.fits || s.m == 0) return s;
    const int64_t m256 = (s.m + 255) / 256, n256 = (s.n + 255) / 256, m128 = (s.m + 127) / 128;
    // Pairs need tiles for most of the 74 of them.  Triangles: 36 tiles (2048 rows) 344 us with pairs, 239 without, 55 (2560 rows) 450 and 439,
    // 136 (4096 rows) two rounds of pairs for 3.6 of single blocks.  B X: 36 tiles (512 x 4608) 167 and 145, 64 (4096 x 1024) 200 and 189,
    // 81 (2300 x 2300) 438 and 462, 96 (3000 x 2000) 311 and 343.
    // Pairs have no tensor memory left for the sums of a long reduction (see LONG).
    s.sym_pair = m256 > 10 && s.n <= kPairLong;
    s.apply_pair = m256 * n256 > 64;
    const bool wide = s.sym_pair || s.apply_pair;
    s.rb = wide ? 4 * m256 : 2 * m128;
    s.cb = wide ? 4 * n256 : (s.n + 127) / 128 * 2;
    s.parts = std::max<int64_t>(1, std::min<int64_t>(kMaxParts, (s.m * s.n + kPartElements - 1) / kPartElements));
    return s;
}
// Blocks that share a tile of a symmetric product of m rows whose reduction is k long: as many as one round of the GPU takes, four
// reduction blocks each at least (33 clusters of four run at once).
int split_of(int64_t m, int64_t k)
{
    const int64_t tiles = ((m + 127) / 128) * ((m + 127) / 128 + 1) / 2, kb = (k + 63) / 64;
    int split = 1;
    while (split < kMaxSplit && 2 * split * tiles <= 132 && 8 * split <= kb) split *= 2;
    return split;
}
size_t scratch_bytes(const Shape &s)
{
    if (s.m == 0) return 0;
    return 3 * (size_t)(s.rb * s.cb) * kBlockBytes + 2 * (size_t)(s.rb * s.rb) * kBlockBytes + (2 + (size_t)s.cb) * (size_t)s.rb * 64 * sizeof(float) +
           kScaleBytes + align256((size_t)s.parts * sizeof(double));
}
// Points an item at its scratch and returns what comes after it.
char *place(NsItem &it, const Shape &s, char *p)
{
    auto take = [&](size_t bytes) { char *at = p; p += bytes; return at; };
    const size_t xs = (size_t)(s.rb * s.cb) * kBlockBytes, as = (size_t)(s.rb * s.rb) * kBlockBytes;
    it.x[0] = reinterpret_cast<uint16_t *>(take(xs));
    it.x[1] = reinterpret_cast<uint16_t *>(take(xs));
    it.lo = reinterpret_cast<uint16_t *>(take(xs));
    it.A = reinterpret_cast<uint16_t *>(take(as));
    it.B = reinterpret_cast<uint16_t *>(take(as));
    it.alpha = reinterpret_cast<float *>(take((size_t)s.rb * 64 * sizeof(float)));
    it.beta = reinterpret_cast<float *>(take((size_t)s.rb * 64 * sizeof(float)));
    it.squares = reinterpret_cast<float *>(take((size_t)s.cb * (size_t)s.rb * 64 * sizeof(float)));
    it.scale = reinterpret_cast<float2 *>(take(kScaleBytes));
    it.part = reinterpret_cast<double *>(take(align256((size_t)s.parts * sizeof(double))));
    it.m = (int)s.m; it.n = (int)s.n; it.rb = (int)s.rb; it.cb = (int)s.cb; it.parts = (int)s.parts;
    it.sym_pair = s.sym_pair; it.apply_pair = s.apply_pair;
    it.count = s.m * s.n;
    return p;
}

// The matrices of P that a kernel serves, `units` of each in one list: by falling split, so that no tile's blocks straddle two
// clusters, then longest reductions first, so that the last tiles are short ones.
template <typename Pick, typename Split, typename Units> bool select(const NsParams &P, NsParams &to, Pick pick, Split split, Units units)
{
    memcpy(reinterpret_cast<char *>(&to) + sizeof(to.item), reinterpret_cast<const char *>(&P) + sizeof(P.item), sizeof(P) - sizeof(P.item));
    to.count = 0;
    for (int t = 0; t < P.count; ++t) {
        if (!pick(P.item[t])) continue;
        NsItem &it = to.item[to.count++];
        it = P.item[t];
        it.split = split(it);
    }
    std::sort(to.item, to.item + to.count, [](const NsItem &a, const NsItem &b) {
        return a.split != b.split ? a.split > b.split : a.n != b.n ? a.n > b.n : a.m > b.m;
    });
    int64_t first = 0;
    for (int t = 0; t < to.count; ++t) {
        to.item[t].first = (int)first;
        first += units(to.item[t]) * to.item[t].split;
        if (first >= 1ll << 31) return false;
    }
    to.units = (int)first;
    return true;
}

template <typename... KArgs, typename... Args>
cudaError_t launch_clusters(void (*kernel)(KArgs...), int grid, int cluster, size_t smem, cudaStream_t s, const Args &...args)
{
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kNsThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <typename Kernel> int allow_smem(Kernel kernel, size_t bytes, bool &done)
{
    if (!done) TWN_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    done = true;
    return TWN_OK;
}
template <int PHASE> int launch_pair(const NsParams &P, const CUtensorMap (&map)[2], const twn_device_info &dev, cudaStream_t s)
{
    static bool done[64] = {false};
    const size_t smem = sizeof(PairSmem) + 1024;
    const int rc = allow_smem(ns_pair_kernel<PHASE>, smem, done[dev.ordinal]);
    if (rc != TWN_OK) return rc;
    TWN_CUDA_OK(launch_clusters(ns_pair_kernel<PHASE>, 2 * std::min(P.units, dev.sm_count / 2), 2, smem, s, map[0], map[1], P));
    return TWN_OK;
}
template <int PHASE, int STAGES, bool LONG> int launch_tile(const NsParams &P, int grid, int cluster, const twn_device_info &dev, cudaStream_t s)
{
    static bool done[64] = {false};
    const size_t smem = sizeof(TileSmem<STAGES>) + 1024;
    const int rc = allow_smem(ns_tile_kernel<PHASE, STAGES, LONG>, smem, done[dev.ordinal]);
    if (rc != TWN_OK) return rc;
    TWN_CUDA_OK(launch_clusters(ns_tile_kernel<PHASE, STAGES, LONG>, grid, cluster, smem, s, P, cluster > 1));
    return TWN_OK;
}
template <int PHASE> int launch_tile(const NsParams &P, const twn_device_info &dev, cudaStream_t s)
{
    int cluster = 1;
    if (PHASE != kApply)
        for (int t = 0; t < P.count; ++t) cluster = std::max(cluster, P.item[t].split);
    const int grid = (P.units + cluster - 1) / cluster * cluster;
    if constexpr (PHASE == kGram) {
        bool chunks = false;
        for (int t = 0; t < P.count; ++t) chunks |= (P.item[t].n + 63) / 64 > (int64_t)kChunk * P.item[t].split;
        if (chunks) return grid <= dev.sm_count ? launch_tile<PHASE, 6, true>(P, grid, cluster, dev, s) : launch_tile<PHASE, 3, true>(P, grid, cluster, dev, s);
    }
    return grid <= dev.sm_count ? launch_tile<PHASE, 6, false>(P, grid, cluster, dev, s) : launch_tile<PHASE, 3, false>(P, grid, cluster, dev, s);
}

// All blocks of the workspace as one matrix of 128-byte rows, in copies of 128 and of 64 of them.
int make_maps(CUtensorMap (&map)[2], void *base, size_t bytes)
{
    auto encode = twn_detail::encode_fn();
    TWN_REQUIRE(encode != nullptr, TWN_ERR_CUDA);
    const cuuint64_t dims[2] = {64, (cuuint64_t)(bytes / 128)}, strides[1] = {128};
    const cuuint32_t ones[2] = {1, 1};
    for (int k = 0; k < 2; ++k) {
        const cuuint32_t box[2] = {64, k == 0 ? 128u : 64u};
        TWN_REQUIRE(encode(&map[k], CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS,
                    TWN_ERR_CUDA);
    }
    return TWN_OK;
}

// Where every matrix of the call is small: one launch for all of it (64 x 576 113 us as fifteen products, see orthogonalize_small.cu).
// In a call with larger ones they ride along in the launches of those.
bool all_small(const NsParams &P, int steps)
{
    for (int t = 0; t < P.count; ++t)
        if (P.item[t].m > twn_detail::kNsSmallM || P.item[t].n > twn_detail::kNsSmallN) return false;
    return steps <= twn_detail::kNsSmallSteps;
}
int run_small(const NsParams &P, int steps, cudaStream_t s)
{
    twn_detail::NsSmallParams S = {};
    S.count = P.count;
    S.steps = steps;
    S.look_ahead = P.look_ahead;
    S.momentum = P.momentum;
    S.eps = P.eps;
    S.status = P.status;
    for (int t = 0; t < P.count; ++t) {
        const NsItem &it = P.item[t];
        static_assert(2 * 4 * kBlockBytes >= twn_detail::kNsSmallScratch, "A and B, one after the other, hold the small path's scratch");
        S.item[t] = {{it.G, it.dW, it.V, it.O, it.m, it.n, it.out_scale, it.g_bf16, it.o_bf16, it.tall, it.vec_in, it.vec_out}, it.A};
    }
    return twn_detail::ns_small(S, s);
}

// What a call writes lies apart from all else that it reads or writes: the matrices of a call are worked on at the same time.
struct Extent {
    const char *begin, *end;
    bool written;
};
struct Extents {
    Extent e[3 * kMaxItems + 1];
    int n = 0;
    void add(const void *p, size_t bytes, bool written) { e[n++] = {static_cast<const char *>(p), static_cast<const char *>(p) + bytes, written}; }
    bool apart()
    {
        std::sort(e, e + n, [](const Extent &a, const Extent &b) { return a.begin < b.begin; });
        const char *any = nullptr, *written = nullptr;       // ends of what begins before
        for (int i = 0; i < n; ++i) {
            if (e[i].begin < (e[i].written ? any : written)) return false;
            any = std::max(any, e[i].end);
            if (e[i].written) written = std::max(written, e[i].end);
        }
        return true;
    }
};

// The items of P are placed from `base` on, within `bytes`.
int run_steps(NsParams &P, int steps, char *base, size_t bytes, Extents &extents, cudaStream_t s)
{
    if (all_small(P, steps)) {
        TWN_REQUIRE(extents.apart(), TWN_ERR_INVALID_ARG);
        return run_small(P, steps, s);
    }
    P.base = reinterpret_cast<const uint16_t *>(base);
    P.steps = steps;
    enum { kNorm, kStartList, kSymPair, kGramTile, kSquareTile, kApplyPair, kApplyTile, kLists };
    NsParams list[kLists];
    auto all = [](const NsItem &) { return true; };
    auto sym_pair = [](const NsItem &it) { return it.sym_pair != 0; };
    auto sym_tile = [](const NsItem &it) { return it.sym_pair == 0; };
    auto one = [](const NsItem &) { return 1; };
    auto triangle = [](int64_t n) { return n * (n + 1) / 2; };
    auto tiles = [&](const NsItem &it) { return triangle(it.rb / 2); };
    const bool fits = select(P, list[kNorm], all, one, [](const NsItem &it) { return (int64_t)it.parts; }) &&
        select(P, list[kStartList], all, one, [](const NsItem &it) { return (int64_t)it.rb * it.cb; }) &&
        select(P, list[kSymPair], sym_pair, one, [&](const NsItem &it) { return triangle(it.rb / 4); }) &&
        select(P, list[kGramTile], sym_tile, [](const NsItem &it) { return split_of(it.m, it.n); }, tiles) &&
        select(P, list[kSquareTile], sym_tile, [](const NsItem &it) { return split_of(it.m, it.m); }, tiles) &&
        select(P, list[kApplyPair], [](const NsItem &it) { return it.apply_pair != 0; }, one, [](const NsItem &it) { return (int64_t)(it.rb / 4) * (it.cb / 4); }) &&
        select(P, list[kApplyTile], [](const NsItem &it) { return it.apply_pair == 0; }, one, [](const NsItem &it) { return (int64_t)(it.rb / 2) * (it.cb / 2); });
    TWN_REQUIRE(fits && bytes / 128 < (1ull << 31), TWN_ERR_TOO_LARGE);
    TWN_REQUIRE(extents.apart(), TWN_ERR_INVALID_ARG);
    twn_device_info dev;
    int rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    CUtensorMap map[2];
    if (list[kSymPair].count + list[kApplyPair].count > 0 && (rc = make_maps(map, base, bytes)) != TWN_OK) return rc;
    TWN_CUDA_OK(twn_launch_small(ns_norm_kernel, std::min(list[kNorm].units, dev.sm_count * 8), kSweepBlock, 0, s, list[kNorm]));
    TWN_CUDA_OK(twn_launch_small(ns_start_kernel, std::min(list[kStartList].units, dev.sm_count * 8), kSweepBlock, 0, s, list[kStartList]));
    for (int step = 0; step < steps; ++step) {
        for (NsParams &l : list) { l.step = step; l.last = step + 1 == steps; }
        if (list[kSymPair].count && (rc = launch_pair<kGram>(list[kSymPair], map, dev, s)) != TWN_OK) return rc;
        if (list[kGramTile].count && (rc = launch_tile<kGram>(list[kGramTile], dev, s)) != TWN_OK) return rc;
        if (list[kSymPair].count && (rc = launch_pair<kSquare>(list[kSymPair], map, dev, s)) != TWN_OK) return rc;
        if (list[kSquareTile].count && (rc = launch_tile<kSquare>(list[kSquareTile], dev, s)) != TWN_OK) return rc;
        if (list[kApplyPair].count && (rc = launch_pair<kApply>(list[kApplyPair], map, dev, s)) != TWN_OK) return rc;
        if (list[kApplyTile].count && (rc = launch_tile<kApply>(list[kApplyTile], dev, s)) != TWN_OK) return rc;
    }
    return TWN_OK;
}

constexpr double kMinEps = 1e-30;            // the factor of the first step stays in the range of fp32

int check_shape(int64_t rows, int64_t cols)
{
    TWN_REQUIRE(rows >= 0 && cols >= 0, TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(rows == 0 || cols == 0 || shape_of(rows, cols).fits, TWN_ERR_TOO_LARGE);
    return TWN_OK;
}
template <typename Item> size_t items_bytes(const Item *items, int count, bool output)
{
    if (count < 0 || count > kMaxItems || (count > 0 && items == nullptr)) return 0;
    size_t bytes = 256;
    for (int t = 0; t < count; ++t) {
        if (check_shape(items[t].rows, items[t].cols) != TWN_OK) return 0;
        if (items[t].rows == 0 || items[t].cols == 0) continue;
        bytes += scratch_bytes(shape_of(items[t].rows, items[t].cols));
        if (output) bytes += align256((size_t)(items[t].rows * items[t].cols) * sizeof(float));
    }
    return bytes;
}

}  // namespace

extern "C" size_t twn_orthogonalize_workspace_bytes(const twn_orthogonalize_item_t *items, int count)
{
    return items_bytes(items, count, false);
}

extern "C" int twn_orthogonalize_batch(const twn_orthogonalize_item_t *items, int count, int steps, double eps, void *workspace,
                                       size_t workspace_bytes, int32_t *dev_status, twn_stream_t stream)
{
    TWN_REQUIRE(count >= 0 && count <= kMaxItems && steps >= 1 && steps <= kMaxSteps, TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(std::isfinite(eps) && eps >= kMinEps && eps <= 1e30, TWN_ERR_INVALID_ARG);
    if (count == 0) return TWN_OK;
    TWN_REQUIRE(items != nullptr && workspace != nullptr, TWN_ERR_INVALID_ARG);
    NsParams P = {};
    Extents extents;
    char *p = static_cast<char *>(workspace);
    for (int t = 0; t < count; ++t) {
        const twn_orthogonalize_item_t &in = items[t];
        const int rc = check_shape(in.rows, in.cols);
        if (rc != TWN_OK) return rc;
        for (int d : {in.g_dtype, in.o_dtype}) TWN_REQUIRE(d == TWN_F32 || d == TWN_BF16, TWN_ERR_INVALID_ARG);
        if (in.rows == 0 || in.cols == 0) continue;
        TWN_REQUIRE(in.G != nullptr && in.O != nullptr, TWN_ERR_INVALID_ARG);
        TWN_REQUIRE(twn_aligned(in.G, in.g_dtype == TWN_BF16 ? 2 : 4) && twn_aligned(in.O, in.o_dtype == TWN_BF16 ? 2 : 4), TWN_ERR_MISALIGNED);
        NsItem &it = P.item[P.count++];
        p = place(it, shape_of(in.rows, in.cols), p);
        it.G = in.G; it.O = in.O;
        it.g_bf16 = in.g_dtype == TWN_BF16; it.o_bf16 = in.o_dtype == TWN_BF16;
        it.tall = in.rows > in.cols;
        it.vec_in = twn_aligned(in.G, 16);
        it.vec_out = twn_aligned(in.O, 16) && in.cols % 8 == 0;      // rows of O on 16-byte boundaries, in runs of eight
        it.out_scale = 1.0f;
        // in place, or else apart
        if (in.G != in.O || it.g_bf16 != it.o_bf16) extents.add(in.G, it.count * (it.g_bf16 ? 2 : 4), false);
        extents.add(in.O, it.count * (it.o_bf16 ? 2 : 4), true);
    }
    const size_t need = twn_orthogonalize_workspace_bytes(items, count);
    TWN_REQUIRE(workspace_bytes >= need, TWN_ERR_WORKSPACE);
    TWN_REQUIRE(twn_aligned(workspace, 256) && twn_aligned(dev_status, 4), TWN_ERR_MISALIGNED);
    if (P.count == 0) return TWN_OK;
    P.eps = (float)eps;
    P.status = dev_status;
    extents.add(workspace, need, true);
    return run_steps(P, steps, static_cast<char *>(workspace), need, extents, twn_cu(stream));
}

extern "C" size_t twn_muon_workspace_bytes(const twn_muon_item_t *items, int count)
{
    const size_t bytes = items_bytes(items, count, true);
    return bytes ? bytes + align256(twn_ternarize_batch_workspace_bytes(count)) : 0;
}

extern "C" int twn_muon_update_batch(const twn_muon_item_t *items, int count, float lr, float momentum, float weight_decay, int look_ahead,
                                     int steps, double eps, double delta_factor, void *workspace, size_t workspace_bytes,
                                     int32_t *dev_status, twn_stream_t stream)
{
    TWN_REQUIRE(count >= 0 && count <= kMaxItems && steps >= 1 && steps <= kMaxSteps, TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(std::isfinite(eps) && eps >= kMinEps && eps <= 1e30, TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(lr == lr && momentum == momentum && weight_decay == weight_decay && (look_ahead == 0 || look_ahead == 1), TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(delta_factor >= 0.0 && delta_factor == delta_factor, TWN_ERR_INVALID_ARG);
    if (count == 0) return TWN_OK;
    TWN_REQUIRE(items != nullptr && workspace != nullptr, TWN_ERR_INVALID_ARG);
    NsParams P = {};
    Extents extents;
    twn_sgd_item_t apply[kMaxItems];
    char *p = static_cast<char *>(workspace);
    void *const sweep_ws = p;
    const size_t sweep_bytes = twn_ternarize_batch_workspace_bytes(count);
    p += align256(sweep_bytes);
    for (int t = 0; t < count; ++t) {
        const twn_muon_item_t &in = items[t];
        const int rc = check_shape(in.rows, in.cols);
        if (rc != TWN_OK) return rc;
        TWN_REQUIRE(twn_aligned(in.W, 16) && twn_aligned(in.dW, 16) && twn_aligned(in.V, 16) && twn_aligned(in.stats_next, 8), TWN_ERR_MISALIGNED);
        apply[t] = {in.W, nullptr, nullptr, in.rows * in.cols, in.stats_next};
        if (in.rows == 0 || in.cols == 0) continue;
        TWN_REQUIRE(in.W != nullptr && in.dW != nullptr && in.V != nullptr, TWN_ERR_INVALID_ARG);
        NsItem &it = P.item[P.count++];
        const Shape s = shape_of(in.rows, in.cols);
        p = place(it, s, p);
        it.dW = in.dW; it.V = in.V; it.O = p;
        extents.add(in.W, it.count * sizeof(float), true);
        extents.add(in.dW, it.count * sizeof(float), false);
        extents.add(in.V, it.count * sizeof(float), true);
        p += align256((size_t)(s.m * s.n) * sizeof(float));
        it.tall = in.rows > in.cols;
        it.vec_in = 1;
        it.vec_out = in.cols % 8 == 0;
        it.out_scale = in.rows > in.cols ? (float)std::sqrt((double)in.rows / (double)in.cols) : 1.0f;
        apply[t].dW = static_cast<const float *>(it.O);      // the whole update: a sweep without a momentum
    }
    const size_t need = twn_muon_workspace_bytes(items, count);
    TWN_REQUIRE(workspace_bytes >= need, TWN_ERR_WORKSPACE);
    TWN_REQUIRE(twn_aligned(workspace, 256) && twn_aligned(dev_status, 4), TWN_ERR_MISALIGNED);
    P.eps = (float)eps;
    P.momentum = momentum;
    P.look_ahead = look_ahead;
    P.status = dev_status;
    if (P.count > 0) {
        extents.add(workspace, need, true);
        const int rc = run_steps(P, steps, static_cast<char *>(workspace), need, extents, twn_cu(stream));
        if (rc != TWN_OK) return rc;
    }
    return twn_detail::apply_updates(apply, count, lr, weight_decay, delta_factor, sweep_ws, sweep_bytes, stream);
}
