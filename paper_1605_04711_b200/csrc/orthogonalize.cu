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
// for a matrix of rank 32, 2e-3 for rank one, where a plain bf16 iteration is off by 1e-2, 0.2 and 1.  X starts at 256 times its value (its elements are near 1/sqrt(m n)), which the first step takes out.
//
// Layout.  X, A and B live in the workspace as blocks of 64x64 fp16 (8 KB), in the 128-byte swizzle that the tensor core
// wants, the row blocks of a column block one after the other.  A tile of 128 rows by 64 columns is then 16 KB in a row, one
// bulk copy, K-major; and the same blocks serve as the MN-major operand of B X, whose reduction runs over the rows of X.
// No tensor maps, and the blocks are padded with zeros, so ragged sizes need no special code.
//
// A and B are symmetric: only tiles on or below the diagonal are computed, and written twice.
//
// One launch per product, for up to 32 matrices at once (their tiles in one list):
//   warp 0     bulk copies into a ring of four 48 KB stages       warp 1   one MMA-issuing thread, 128x256 tiles
//   warps 2-9  epilogue, two per tensor-memory lane quadrant; two accumulators, so it runs beside the next tile
#include <algorithm>
#include <cmath>
#include <cstddef>

#include <cuda_fp16.h>

#include "common.cuh"
#include "tc_ptx.cuh"

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kStart = 256.0f;             // X of the first step is this much larger
constexpr int kMaxItems = 32;
constexpr int kBlockBytes = 8192, kBlockHalves = kBlockBytes / 2;
constexpr int kStages = 4, kABytes = 2 * kBlockBytes, kBBytes = 4 * kBlockBytes, kStageBytes = kABytes + kBBytes;
constexpr int kAccCols = 256;
constexpr int kEpiWarps = 8;
constexpr int kNsThreads = 32 * (2 + kEpiWarps);
constexpr int kMaxParts = 148;               // of a matrix's sum of squares
constexpr long long kPartElements = 16384;
constexpr int kSweepBlock = 256;

enum { kGram = 0, kSquare = 1, kApply = 2 };

struct NsItem {
    const void *G;               // the update; NULL for Muon, whose update is
    const float *dW;             //   V, or dW + momentum V (look ahead), with
    float *V;                    //   V = momentum V + dW, which the first sweep writes
    void *O;
    uint16_t *x[2], *lo, *A, *B; // blocks
    float *alpha, *beta;         // diagonals
    float *squares;              // [2 cb][64 rb]: sums of squares of 32 elements of a row of X
    double *part;                // sums of squares
    long long count;             // elements
    int m, n, rb, cb;            // shorter and longer side; row blocks of X (even) and column blocks
    int parts, part_first, block_first, sym_first, apply_first;
    float out_scale;
    uint8_t g_bf16, o_bf16, tall;
};

struct NsParams {
    NsItem item[kMaxItems];
    int count, units, step, last;
    float momentum, eps;
    int look_ahead;
    int32_t *status;
};

enum { kPartList, kBlockList, kSymList, kApplyList };
template <int LIST> __device__ __forceinline__ int first_of(const NsItem &it)
{
    return LIST == kPartList ? it.part_first : LIST == kBlockList ? it.block_first : LIST == kSymList ? it.sym_first : it.apply_first;
}
template <int LIST> __device__ __forceinline__ int item_of(const NsParams &P, int unit)
{
    int t = 0;
    while (t + 1 < P.count && unit >= first_of<LIST>(P.item[t + 1])) ++t;
    return t;
}

// Block (R, C) of a matrix of rb row blocks.
__device__ __forceinline__ size_t block_at(int R, int C, int rb) { return ((size_t)C * rb + R) * kBlockHalves; }
// Element (r, c) of a block: rows of 128 bytes, their 16-byte pieces exchanged by the row's number modulo 8.
__device__ __forceinline__ int in_block(int r, int c) { return r * 64 + ((((c >> 3) ^ r) & 7) << 3) + (c & 7); }

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

// Sum of squares of every matrix, in fp64 and in a fixed order; for Muon the momentum is updated on the way.
__global__ void __launch_bounds__(kSweepBlock) ns_norm_kernel(const __grid_constant__ NsParams P)
{
    __shared__ double red[kSweepBlock / 32];
    pdl_begin();
    for (int u = blockIdx.x; u < P.units; u += gridDim.x) {
        const NsItem &it = P.item[item_of<kPartList>(P, u)];
        const int part = u - it.part_first;
        const long long per = ((it.count + it.parts - 1) / it.parts + 1023) / 1024 * 1024;
        const long long end = min(it.count, (part + 1) * per);
        double s = 0.0;
#pragma unroll 4
        for (long long i = part * per + threadIdx.x; i < end; i += kSweepBlock) {
            double g;
            if (it.V) {
                const float d = it.dW[i], v = __fadd_rn(__fmul_rn(P.momentum, it.V[i]), d);
                it.V[i] = v;
                g = muon_update(P, v, d);
            } else {
                g = element(it, P, i);
            }
            s += g * g;
        }
        s = block_sum(s, red);
        if (threadIdx.x == 0) it.part[part] = s;
    }
}

// X of the first step, a block of 64x64 at a time: normalised, split into two fp16 numbers, padded with zeros.
__global__ void __launch_bounds__(kSweepBlock) ns_start_kernel(const __grid_constant__ NsParams P)
{
    __shared__ double red[kSweepBlock / 32];
    __shared__ float tile[64][65];
    pdl_begin();
    for (int u = blockIdx.x; u < P.units; u += gridDim.x) {
        const NsItem &it = P.item[item_of<kBlockList>(P, u)];
        const int b = u - it.block_first, R = b % it.rb, C = b / it.rb;
        double s = 0.0;
        for (int p = threadIdx.x; p < it.parts; p += kSweepBlock) s += it.part[p];
        const double norm = sqrt(block_sum(s, red));
        if (b == 0 && threadIdx.x == 0 && P.status && !isfinite(norm)) atomicMin(P.status, (int)TWN_ERR_NONFINITE);
        // in two factors, so that neither leaves the range of fp32
        const float pre = norm > 1e18 ? 0x1p-100f : 1.0f;
        const float factor = norm == 0.0 ? 0.0f : (float)((double)kStart / (fmax(norm, (double)P.eps) * (double)pre));
        const float nan = norm == norm ? 0.0f : __uint_as_float(0x7FC00000u);      // fmax drops a NaN
        const int r0 = 64 * R, c0 = 64 * C;
        // rows of G along the threads of a warp
        for (int e = threadIdx.x; e < 4096; e += kSweepBlock) {
            const int i = e >> 6, j = e & 63;
            const int r = r0 + (it.tall ? j : i), c = c0 + (it.tall ? i : j);
            float v = 0.0f;
            if (r < it.m && c < it.n) v = element(it, P, it.tall ? (long long)c * it.m + r : (long long)r * it.n + c) * pre * factor + nan;
            tile[it.tall ? j : i][it.tall ? i : j] = v;
        }
        __syncthreads();
        uint16_t *const hi = it.x[0] + block_at(R, C, it.rb), *const lo = it.lo + block_at(R, C, it.rb);
        for (int e = threadIdx.x; e < 2048; e += kSweepBlock) {
            const int r = e >> 5, c = 2 * (e & 31);
            const float v0 = tile[r][c], v1 = tile[r][c + 1];
            const __half2 h = __floats2half2_rn(v0, v1);
            const float2 back = __half22float2(h);
            const __half2 l = __floats2half2_rn(v0 - back.x, v1 - back.y);
            *reinterpret_cast<__half2 *>(hi + in_block(r, c)) = h;
            *reinterpret_cast<__half2 *>(lo + in_block(r, c)) = l;
        }
        if (threadIdx.x < 128) {
            const int r = threadIdx.x & 63, half = threadIdx.x >> 6;
            float q = 0.0f;
            for (int c = 32 * half; c < 32 * half + 32; ++c) q = fmaf(tile[r][c], tile[r][c], q);
            it.squares[(size_t)(2 * C + half) * (64 * it.rb) + r0 + r] = q;
        }
    }
}

struct __align__(1024) NsSmem {
    uint8_t ring[kStages][kStageBytes];
    unsigned long long full[kStages], empty[kStages], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    volatile int abort_flag;
};

__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, void *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

// D[tmem] (+)= A[smem] B[smem]^T, fp16, issued by the calling thread alone.
__device__ __forceinline__ void ns_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc)
        : "memory");
}

// A tile: 128 rows from block row 2 i on, `nb` (at most 4) blocks of columns from block 4 J on, a reduction of kb blocks.
struct Tile {
    int i, J, nb, kb;
};
template <int PHASE> __device__ __forceinline__ Tile tile_of(const NsItem &it, int u)
{
    Tile t;
    const int pairs = it.rb >> 1;                      // row tiles
    if (PHASE == kApply) {
        u -= it.apply_first;
        t.i = u % pairs;
        t.J = u / pairs;
        t.nb = min(4, it.cb - 4 * t.J);
        t.kb = (it.m + 63) >> 6;
    } else {
        // row tiles 2p and 2p + 1 have p + 1 tiles each, on or below the diagonal
        u -= it.sym_first;
        int p = (int)((sqrtf(4.0f * (float)u + 1.0f) - 1.0f) * 0.5f);
        while (p * (p + 1) > u) --p;
        while ((p + 1) * (p + 2) <= u) ++p;
        const int rem = u - p * (p + 1);
        t.i = 2 * p + (rem > p);
        t.J = rem > p ? rem - p - 1 : rem;
        t.nb = min(4, it.rb - 4 * t.J);
        t.kb = PHASE == kGram ? it.cb : (it.m + 63) >> 6;
    }
    return t;
}

__device__ __forceinline__ uint32_t half2_bits(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 half2_of(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

template <int PHASE>
__global__ void __launch_bounds__(kNsThreads, 1) ns_product_kernel(const __grid_constant__ NsParams P)
{
    constexpr int LIST = PHASE == kApply ? kApplyList : kSymList;
    if (gridDim.x <= kPdlBlocks) pdl_launch_dependents();
    extern __shared__ uint8_t smem_raw[];
    NsSmem *sm = reinterpret_cast<NsSmem *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    volatile int *abort_flag = &sm->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(&sm->full[s], 1); mbar_init(&sm->empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&sm->acc_full[s], 1); mbar_init(&sm->acc_empty[s], kEpiWarps); }
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
    pdl_wait();
    const uint32_t tmem = sm->tmem_base;
    const int cur = P.step & 1;

    if (warp == 0) {
        if (elect_one()) {
            uint32_t s = 0, ph = 0;
            bool ok = true;
            for (int u = blockIdx.x; u < P.units && ok; u += gridDim.x) {
                const NsItem &it = P.item[item_of<LIST>(P, u)];
                const Tile t = tile_of<PHASE>(it, u);
                const uint16_t *const src_a = PHASE == kGram ? it.x[cur] : PHASE == kSquare ? it.A : it.B;
                const uint16_t *const src_b = PHASE == kSquare ? it.A : it.x[cur];
                const uint32_t b_bytes = (uint32_t)t.nb * kBlockBytes;
                for (int k = 0; k < t.kb; ++k) {
                    uint8_t *const st = sm->ring[s];
                    if (!mbar_wait(&sm->empty[s], ph ^ 1u, abort_flag, P.status, 20)) { ok = false; break; }
                    mbar_expect_tx(&sm->full[s], kABytes + b_bytes);
                    bulk_load(st, src_a + block_at(2 * t.i, k, it.rb), kABytes, &sm->full[s]);
                    if (PHASE == kApply) {
                        for (int j = 0; j < t.nb; ++j)
                            bulk_load(st + kABytes + j * kBlockBytes, src_b + block_at(k, 4 * t.J + j, it.rb), kBlockBytes, &sm->full[s]);
                    } else {
                        bulk_load(st + kABytes, src_b + block_at(4 * t.J, k, it.rb), b_bytes, &sm->full[s]);
                    }
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            uint32_t s = 0, ph = 0, lu = 0;
            bool ok = true;
            const uint32_t ring = smem_u32(sm->ring);
            const uint64_t a0 = smem_desc_sw128(ring);
            const uint64_t b0 = PHASE == kApply ? smem_desc_mn_sw128(ring + kABytes, kBlockBytes) : smem_desc_sw128(ring + kABytes);
            constexpr uint64_t kStageStep = kStageBytes >> 4;
            constexpr uint64_t kBStep = PHASE == kApply ? (16 * 128) >> 4 : 32 >> 4;      // 16 rows of the reduction, or 16 columns
            for (int u = blockIdx.x; u < P.units && ok; u += gridDim.x, ++lu) {
                const NsItem &it = P.item[item_of<LIST>(P, u)];
                const Tile t = tile_of<PHASE>(it, u);
                // fp16 operands, fp32 accumulator, B MN-major where it is X
                const uint32_t idesc = (1u << 4) | (PHASE == kApply ? 1u << 16 : 0u) | ((uint32_t)(t.nb * 8) << 17) | (8u << 24);
                if (!mbar_wait(&sm->acc_empty[lu & 1], ((lu >> 1) & 1u) ^ 1u, abort_flag, P.status, 0)) break;
                tc_fence_after();
                const uint32_t d = tmem + (lu & 1) * kAccCols;
                for (int k = 0; k < t.kb; ++k) {
                    if (!mbar_wait(&sm->full[s], ph, abort_flag, P.status, 0)) { ok = false; break; }
                    tc_fence_after();
                    const uint64_t a = a0 + s * kStageStep, b = b0 + s * kStageStep;
                    ns_mma(d, a, b, idesc, k > 0);
                    ns_mma(d, a + 2, b + kBStep, idesc, 1u);
                    ns_mma(d, a + 4, b + 2 * kBStep, idesc, 1u);
                    ns_mma(d, a + 6, b + 3 * kBStep, idesc, 1u);
                    tc_commit(&sm->empty[s]);
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
                if (ok) tc_commit(&sm->acc_full[lu & 1]);
            }
        }
    } else {
        const int q = warp & 3, set = (warp - 2) >> 2;
        uint32_t lu = 0;
        for (int u = blockIdx.x; u < P.units; u += gridDim.x, ++lu) {
            const NsItem &it = P.item[item_of<LIST>(P, u)];
            const Tile t = tile_of<PHASE>(it, u);
            if (!mbar_wait_warp(&sm->acc_full[lu & 1], (lu >> 1) & 1u, abort_flag, P.status, 32)) break;
            tc_fence_after();
            const int r = 128 * t.i + 32 * q + lane;
            const float unscale = P.step == 0 ? 1.0f / kStart : 1.0f;
            const float row_diag = PHASE == kSquare ? it.alpha[r] : PHASE == kApply ? it.beta[r] : 0.0f;
            // a warp has every other chunk of 32 columns
#pragma unroll 1
            for (int ch = set; ch < 2 * t.nb; ch += 2) {
                const int c0 = 256 * t.J + 32 * ch;
                if (PHASE != kApply && (c0 >> 7) > t.i) break;             // above the diagonal: another tile's mirror image
                uint32_t v[32];
                tmem_ld32(tmem + ((uint32_t)(32 * q) << 16) + (lu & 1) * kAccCols + 32 * ch, v);
                tmem_wait_ld(v);
                // this thread's 32 elements of the row: four 16-byte pieces
                const size_t block = block_at(r >> 6, c0 >> 6, it.rb);
                uint16_t *const to = PHASE == kGram ? it.A : PHASE == kSquare ? it.B : it.x[cur ^ 1];
                float f[32];
                if (PHASE == kGram) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]) * (unscale * unscale);
                } else if (PHASE == kSquare) {
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const uint4 w = *reinterpret_cast<const uint4 *>(it.A + block + in_block(r & 63, (c0 & 63) + 8 * p));
                        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int e = 8 * p + 2 * j;
                            const float2 a = half2_of(ws[j]);
                            const float2 al = *reinterpret_cast<const float2 *>(it.alpha + c0 + e);
                            f[e] = kB * a.x + kC * (__uint_as_float(v[e]) + (row_diag + al.x) * a.x);
                            f[e + 1] = kB * a.y + kC * (__uint_as_float(v[e + 1]) + (row_diag + al.y) * a.y);
                        }
                    }
                } else {
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const int at = in_block(r & 63, (c0 & 63) + 8 * p);
                        const uint4 h = *reinterpret_cast<const uint4 *>(it.x[cur] + block + at);
                        const uint4 l = *reinterpret_cast<const uint4 *>(it.lo + block + at);
                        const uint32_t hs[4] = {h.x, h.y, h.z, h.w}, ls[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int e = 8 * p + 2 * j;
                            const float2 x = half2_of(hs[j]), y = half2_of(ls[j]);
                            f[e] = ((kA + row_diag) * (x.x + y.x) + __uint_as_float(v[e])) * unscale;
                            f[e + 1] = ((kA + row_diag) * (x.y + y.y) + __uint_as_float(v[e + 1])) * unscale;
                        }
                    }
                }
                if (PHASE != kApply && (unsigned)(r - c0) < 32u) {
                    // the diagonal, apart: selected without indexing registers by a variable
                    float dia = 0.0f;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (r - c0 == j) {
                            if (PHASE == kSquare) dia = kB * row_diag + kC * (__uint_as_float(v[j]) + row_diag * row_diag);
                            f[j] = 0.0f;
                        }
                    if (PHASE == kGram) {
#pragma unroll 8
                        for (int g = 0; g < 2 * it.cb; ++g) dia += it.squares[(size_t)g * (64 * it.rb) + r];
                        dia *= unscale * unscale;
                    }
                    (PHASE == kGram ? it.alpha : it.beta)[r] = dia;
                }
                if (PHASE == kApply && P.last) {
                    if (r < it.m) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const int c = c0 + j;
                            if (c < it.n) {
                                const long long at = it.tall ? (long long)c * it.m + r : (long long)r * it.n + c;
                                const float o = f[j] * it.out_scale;
                                if (it.o_bf16) static_cast<__nv_bfloat16 *>(it.O)[at] = __float2bfloat16_rn(o);
                                else static_cast<float *>(it.O)[at] = o;
                            }
                        }
                    }
                    continue;
                }
                if (PHASE == kApply) {
                    float sq = 0.0f;
#pragma unroll
                    for (int j = 0; j < 32; ++j) sq = fmaf(f[j], f[j], sq);
                    it.squares[(size_t)(c0 >> 5) * (64 * it.rb) + r] = sq;
                }
                uint32_t h[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) h[j] = half2_bits(f[2 * j], f[2 * j + 1]);
#pragma unroll
                for (int p = 0; p < 4; ++p)
                    *reinterpret_cast<uint4 *>(to + block + in_block(r & 63, (c0 & 63) + 8 * p)) =
                        make_uint4(h[4 * p], h[4 * p + 1], h[4 * p + 2], h[4 * p + 3]);
                if (PHASE == kApply) {
                    uint32_t l[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float2 x = half2_of(h[j]);
                        l[j] = half2_bits(f[2 * j] - x.x, f[2 * j + 1] - x.y);
                    }
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        *reinterpret_cast<uint4 *>(it.lo + block + in_block(r & 63, (c0 & 63) + 8 * p)) =
                            make_uint4(l[4 * p], l[4 * p + 1], l[4 * p + 2], l[4 * p + 3]);
                } else if ((c0 >> 7) < t.i) {
                    // the mirror image
                    const size_t mirror = block_at(c0 >> 6, r >> 6, it.rb);
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        to[mirror + in_block((c0 & 63) + j, r & 63)] = (uint16_t)((j & 1) ? h[j >> 1] >> 16 : h[j >> 1] & 0xFFFFu);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm->acc_empty[lu & 1]);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (sm->abort_flag) {
        // copies and products in flight end well within this
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
size_t align256(size_t v) { return (v + 255) / 256 * 256; }

struct Shape {
    int64_t m, n, rb, cb, parts;
    bool fits;
};
constexpr int64_t kMaxShort = 32768, kMaxLong = 1 << 24;
Shape shape_of(int64_t rows, int64_t cols)
{
    Shape s;
    s.m = std::min(rows, cols);
    s.n = std::max(rows, cols);
    s.fits = s.m <= kMaxShort && s.n <= kMaxLong;
    s.rb = (s.m + 127) / 128 * 2;
    s.cb = (s.n + 63) / 64;
    s.parts = s.fits ? std::max<int64_t>(1, std::min<int64_t>(kMaxParts, (s.m * s.n + kPartElements - 1) / kPartElements)) : 0;
    return s;
}
size_t scratch_bytes(const Shape &s)
{
    if (s.m == 0) return 0;
    return 3 * (size_t)(s.rb * s.cb) * kBlockBytes + 2 * (size_t)(s.rb * s.rb) * kBlockBytes + (2 + 2 * (size_t)s.cb) * (size_t)s.rb * 64 * sizeof(float) +
           align256((size_t)s.parts * sizeof(double));
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
    it.squares = reinterpret_cast<float *>(take(2 * (size_t)s.cb * (size_t)s.rb * 64 * sizeof(float)));
    it.part = reinterpret_cast<double *>(take(align256((size_t)s.parts * sizeof(double))));
    it.m = (int)s.m; it.n = (int)s.n; it.rb = (int)s.rb; it.cb = (int)s.cb; it.parts = (int)s.parts;
    it.count = s.m * s.n;
    return p;
}

template <int PHASE> int launch_product(NsParams &P, int units, const twn_device_info &dev, cudaStream_t s)
{
    static bool attr_set[64] = {false};
    const int smem = (int)sizeof(NsSmem) + 1024;
    if (!attr_set[dev.ordinal]) {
        TWN_CUDA_OK(cudaFuncSetAttribute(ns_product_kernel<PHASE>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        attr_set[dev.ordinal] = true;
    }
    P.units = units;
    TWN_CUDA_OK(twn_launch_pdl(true, ns_product_kernel<PHASE>, std::min(units, dev.sm_count), kNsThreads, (size_t)smem, s, P));
    return TWN_OK;
}

// The items of P are placed; longest reductions first, so that the last tiles are short ones.
int run_steps(NsParams &P, int steps, cudaStream_t s)
{
    std::sort(P.item, P.item + P.count, [](const NsItem &a, const NsItem &b) { return a.n != b.n ? a.n > b.n : a.m > b.m; });
    int64_t parts = 0, blocks = 0, sym = 0, apply = 0;
    for (int t = 0; t < P.count; ++t) {
        NsItem &it = P.item[t];
        it.part_first = (int)parts; it.block_first = (int)blocks; it.sym_first = (int)sym; it.apply_first = (int)apply;
        const int64_t pairs = it.rb / 2, p = pairs / 2;
        parts += it.parts;
        blocks += (int64_t)it.rb * it.cb;
        sym += p * (p + 1) + (pairs % 2 ? p + 1 : 0);
        apply += pairs * ((it.cb + 3) / 4);
    }
    TWN_REQUIRE(blocks < (1ll << 31), TWN_ERR_TOO_LARGE);
    twn_device_info dev;
    int rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    P.units = (int)parts;
    TWN_CUDA_OK(twn_launch_small(ns_norm_kernel, (int)std::min<int64_t>(parts, 148 * 8), kSweepBlock, 0, s, P));
    P.units = (int)blocks;
    TWN_CUDA_OK(twn_launch_small(ns_start_kernel, (int)std::min<int64_t>(blocks, 148 * 8), kSweepBlock, 0, s, P));
    for (P.step = 0; P.step < steps; ++P.step) {
        P.last = P.step + 1 == steps;
        if ((rc = launch_product<kGram>(P, (int)sym, dev, s)) != TWN_OK) return rc;
        if ((rc = launch_product<kSquare>(P, (int)sym, dev, s)) != TWN_OK) return rc;
        if ((rc = launch_product<kApply>(P, (int)apply, dev, s)) != TWN_OK) return rc;
    }
    return TWN_OK;
}

constexpr int kMaxSteps = 32;
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
        it.out_scale = 1.0f;
    }
    TWN_REQUIRE(workspace_bytes >= twn_orthogonalize_workspace_bytes(items, count), TWN_ERR_WORKSPACE);
    TWN_REQUIRE(twn_aligned(workspace, 256) && twn_aligned(dev_status, 4), TWN_ERR_MISALIGNED);
    if (P.count == 0) return TWN_OK;
    P.eps = (float)eps;
    P.status = dev_status;
    return run_steps(P, steps, twn_cu(stream));
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
        p += align256((size_t)(s.m * s.n) * sizeof(float));
        it.tall = in.rows > in.cols;
        it.out_scale = in.rows > in.cols ? (float)std::sqrt((double)in.rows / (double)in.cols) : 1.0f;
        // the update with the orthogonalised matrix as gradient and no momentum; that sweep's V is the matrix itself,
        // every element of which it reads before it writes it
        apply[t].dW = static_cast<const float *>(it.O);
        apply[t].V = static_cast<float *>(it.O);
    }
    TWN_REQUIRE(workspace_bytes >= twn_muon_workspace_bytes(items, count), TWN_ERR_WORKSPACE);
    TWN_REQUIRE(twn_aligned(workspace, 256) && twn_aligned(dev_status, 4), TWN_ERR_MISALIGNED);
    P.eps = (float)eps;
    P.momentum = momentum;
    P.look_ahead = look_ahead;
    P.status = dev_status;
    if (P.count > 0) {
        const int rc = run_steps(P, steps, twn_cu(stream));
        if (rc != TWN_OK) return rc;
    }
    return twn_sgd_update_batch(apply, count, lr, 0.0f, weight_decay, delta_factor, sweep_ws, sweep_bytes, stream);
}
