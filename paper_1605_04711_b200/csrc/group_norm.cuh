// Group norm over groups of channels of an image, channels last, with an activation behind it, forward and backward.
//
//   forward   N = HW C / G values of an image's group:  mean = sum x / N,  var = sum (x - mean)^2 / N,  rstd = 1 / sqrt(var + eps)
//             y = act(z),  z = (x - mean) rstd gamma + beta
//   backward  dz = dy act'(z),  A[c] = sum over the image of dz,  D[c] = sum of dz (x - mean)
//             s = sum over the group's channels of gamma A,  t = sum of gamma D
//             dx = dz rstd gamma - rstd s / N - (x - mean) rstd^3 t / N,  dbeta = sum over the images of A,  dgamma = sum of rstd D
//
// Bound by HBM where the tensors are large.  An image's channels are cut into slabs of whole groups, and a slab's pixels into tiles, a tile
// a block; the blocks of a slab are a cluster.  A thread has V channels (16 bytes of the wider type, where C and the rows
// allow) of every R-th pixel of the tile.
//
//   resident  tiles stay in shared memory, each thread's own vectors by its own asynchronous copies, so that no barrier guards them and every
//             element crosses HBM once in each direction; the blocks' sums meet through distributed shared memory.
//   two reads where a slab is more than a cluster of eight holds: a launch of sums, which writes each tile's to the workspace, and one that reads
//             the tensors again and joins the sums first.
#pragma once

#include <numeric>

#include "layer_norm.cuh"
#include "sweep.cuh"

namespace {

constexpr int kGnThreads = 256;
constexpr int kMaxCluster = 8;
constexpr int kSms = 148;            // that tiles are made for: the workspace is the same on any device, and without one
constexpr int kRun = 64;             // pixels that a thread adds up by themselves: sums of millions of them keep their digits
constexpr size_t kTileTwo = 112 * 1024, kTileMost = 224 * 1024;     // shared memory of a block where there are two an SM, and of one at most
constexpr size_t kTileLeast = 64 * 1024;                            // what small images' blocks grow to

template <> struct Vec<bf16, 2> {
    uint32_t r;
    __device__ void load(const bf16 *p) { r = *reinterpret_cast<const uint32_t *>(p); }
    __device__ void zero() { r = 0u; }
    __device__ void get(float (&f)[2]) const { f[0] = __uint_as_float(r << 16); f[1] = __uint_as_float(r & 0xFFFF0000u); }
};
template <> struct Vec<float, 2> {
    float2 r;
    __device__ void load(const float *p) { r = *reinterpret_cast<const float2 *>(p); }
    __device__ void zero() { r = make_float2(0.f, 0.f); }
    __device__ void get(float (&f)[2]) const { f[0] = r.x; f[1] = r.y; }
};
__device__ __forceinline__ void store(bf16 *p, const float (&f)[2]) { *reinterpret_cast<uint32_t *>(p) = two_bf16(f[0], f[1]); }
__device__ __forceinline__ void store(float *p, const float (&f)[2]) { *reinterpret_cast<float2 *>(p) = make_float2(f[0], f[1]); }

enum { kNone = TWN_ACT_NONE, kRelu = TWN_ACT_RELU, kSilu = TWN_ACT_SILU };

// Quotients of numbers below 2^31 by one that the host knows.
struct Div {
    uint32_t d, m, s;
    Div() = default;
    explicit Div(uint32_t by) : d(by), m(0), s(0)
    {
        while ((1ull << s) < by) ++s;
        m = (uint32_t)(((1ull << 32) * ((1ull << s) - by)) / by + 1);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (__umulhi(n, m) + n) >> s; }
};

// How a call is cut up.
struct Cut {
    long long HW, rows;              // pixels of an image, of a tile
    int C, G, Cg;
    int slab, slabs;                 // channels of a slab; slabs of an image
    int tiles;                       // of a slab
    int pieces;                      // slabs of a group, where a group is more than a slab (the last may have fewer channels); else 1
    int lg_u;                        // channels (their logarithm) that a thread's sums are joined over
    int groups, per, sets;           // groups of a slab (1 for a piece); a group's sets of joined channels; a slab's
    int head;                        // pixels of a thread that its sums' first anchor is the average of
    int R, joint, least;             // pixels of a block at once; of them, those that are joined inside a warp: lanes `least` apart (32 where none are)
    int rows_of_sums;                // rows of threads, or warps where those are joined
    int lg_tile, lg_slab;            // lanes (their logarithms) that join a group's sums, of a tile, of a slab's tiles
    double inv_n;                    // 1 / (HW Cg)
    Div by_tiles, by_slabs, by_vectors, by_group, by_per;
};

// Channels that a thread's sums are joined over before they meet the others': the whole vector inside one group, whole groups
// inside the vector, or single channels.
int joined(int Cg, int V) { return Cg % V == 0 ? V : V % Cg == 0 ? Cg : 1; }

// What a block and a thread have of it.
template <int V> struct Tile {
    long long b, first;              // image; first pixel
    int tile, c0, cs, rows;          // first channel and channels of the slab; pixels
    int VW, R, tx, ty, n;            // vectors of a pixel; pixels at once; the thread's place; its pixels
    int base, rest;                  // pixels of every thread; of those of the first `rest` rows of threads one more
    __device__ __forceinline__ Tile(const Cut &k, unsigned int block)
    {
        const unsigned int s = k.by_tiles(block);
        tile = (int)(block - s * (unsigned)k.tiles);
        const unsigned int image = k.by_slabs(s);
        const int i = (int)(s - image * (unsigned)k.slabs);
        b = image;
        c0 = i * k.slab;
        cs = k.slab;
        VW = cs / V;
        R = k.R;
        if (k.pieces > 1) {
            const int g = i / k.pieces, p = i - g * k.pieces;
            c0 = g * k.Cg + p * k.slab;
            cs = min(k.slab, k.Cg - p * k.slab);
            VW = cs / V;                         // R stays: threads beyond have nothing
            ty = threadIdx.x / (k.slab / V);
            tx = threadIdx.x % (k.slab / V);
        } else {
            ty = (int)k.by_vectors(threadIdx.x);
            tx = threadIdx.x - ty * VW;
        }
        first = (long long)tile * k.rows;
        rows = (int)max(0ll, min(k.rows, k.HW - first));
        base = rows / R;
        rest = rows - base * R;
        n = has() ? base + (ty < rest) : 0;
    }
    __device__ __forceinline__ bool has() const { return ty < R && tx < VW; }
    __device__ __forceinline__ int channel() const { return c0 + tx * V; }
};

// (two bytes, which no asynchronous copy takes, are stored at once)
template <int BYTES> __device__ __forceinline__ void copy_in(uint32_t dst, const void *src)
{
    if (BYTES == 2) asm volatile("st.shared.u16 [%0], %1;" ::"r"(dst), "h"(__ldg(static_cast<const unsigned short *>(src))) : "memory");
    else if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES < 4 ? 4 : BYTES) : "memory");
}
// n vectors of V elements, `step` elements apart, to a thread's slots.
template <typename T, int V> __device__ __forceinline__ void copy_vectors(T *slots, const T *from, long long step, int n)
{
    uint32_t to = smem_u32(slots);
    if (V * sizeof(T) == 2) {
        for (; n >= 8; n -= 8, to += 8 * kGnThreads * V * sizeof(T), from += 8 * step) {
            unsigned short v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __ldg(reinterpret_cast<const unsigned short *>(from + j * step));
#pragma unroll
            for (int j = 0; j < 8; ++j) asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + j * (uint32_t)(kGnThreads * V * sizeof(T))), "h"(v[j]) : "memory");
        }
    }
    for (; n > 0; --n, to += kGnThreads * V * sizeof(T), from += step) copy_in<V * sizeof(T)>(to, from);
}
// A thread's copies are asked for in two shares, and one is worked on while the other is on its way.
constexpr int kShares = 2;
__device__ __forceinline__ int share_end(int n, int q) { return (n * (q + 1) + kShares - 1) / kShares; }
__device__ __forceinline__ void end_share() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void shares_left() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
// work(begin, end) for each share of n, as it comes.
template <int Q = 0, typename Work> __device__ __forceinline__ void as_they_come(int n, int begin, const Work &work)
{
    if constexpr (Q < kShares) {
        shares_left<kShares - 1 - Q>();
        const int end = share_end(n, Q);
        work(begin, end);
        as_they_come<Q + 1>(n, end, work);
    }
}

// Sums over 2^lg neighbouring lanes, in all of them.
template <typename T> __device__ __forceinline__ T all_sum(T v, int lg)
{
    for (int o = (1 << lg) >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// What the blocks of a cluster send each other, before they meet at its barrier.  (With an arrival on a barrier in the receiver's memory behind every store, each with a
// fence of its own, 64 x 12544 x 64 took 61 us forward for 57 at the time.)
__device__ __forceinline__ void send(const void *own, int rank, float a)
{
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_smem(own, rank)), "f"(a) : "memory");
}

// V numbers of fp32 from p on, four at a time where they lie on 16 bytes.
template <int V> __device__ __forceinline__ void load_floats(float (&f)[V], const float *p)
{
    if (V % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
        for (int i = 0; i + 4 <= V; i += 4) {
            const float4 v = __ldg(reinterpret_cast<const float4 *>(p + i));
            f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = __ldg(p + i);
    }
}

// SiLU of z below this counts as that of this, -1.4e-36: exp(87) is still a number, and 1 / (1 + exp(87)) one of full digits.
constexpr float kLeastZ = -87.0f, kMinusLog2e = -1.4426950408889634f;
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float reciprocal(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// (a NaN stays one)
__device__ __forceinline__ float at_least(float x, float least)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(least));
    return r;
}
// exp(-z) and 1 / (1 + exp(-z)) of two neighbouring channels of J pixels, z at least kLeastZ.  With two pixels one reciprocal serves a channel of both, whose z are NaN together, and
// never two channels, which may be of different groups (forward, 64 x 3136 x 256 bf16: 54.4 us, with one for each z 57.4); the factor of 2^-126 keeps the product of
// two sums from 1 to 2^126 inside the numbers.
template <int J> __device__ __forceinline__ void sigmoids(const two_f32 (&z)[J], two_f32 (&e)[J], two_f32 (&f)[J])
{
    const two_f32 one = two(1.0f, 1.0f), scale = two(0x1p-126f, 0x1p-126f);
    two_f32 s[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        float t0, t1;
        each(mul2(z[j], two(kMinusLog2e, kMinusLog2e)), t0, t1);
        e[j] = two(ex2(t0), ex2(t1));
        s[j] = j == 1 ? fma2(e[j], scale, scale) : add2(e[j], one);
    }
    float p0, p1;
    each(J == 2 ? mul2(s[0], s[J - 1]) : s[0], p0, p1);
    f[0] = two(reciprocal(p0), reciprocal(p1));
    if (J == 2) {
        f[J - 1] = mul2(mul2(f[0], s[0]), scale);
        f[0] = mul2(f[0], s[J - 1]);
    }
}
__device__ __forceinline__ two_f32 at_least2(two_f32 z, float least)
{
    float a, b;
    each(z, a, b);
    return two(at_least(a, least), at_least(b, least));
}

bool is_act(int a) { return a == TWN_ACT_NONE || a == TWN_ACT_RELU || a == TWN_ACT_SILU; }

// Vectors of V channels fit the groups: whole groups make whole vectors within a block's threads, or a group is many vectors.
bool vectors_fit(int Cg, int V) { return std::lcm((long long)Cg, (long long)V) / V <= kGnThreads || Cg % V == 0; }

// The widest vectors, of `most` elements or fewer, that C, the groups and the rows of all tensors (which rows(V) looks at) are made of.  (8 x 4096 pixels bf16 with SiLU: 924
// channels in fours 49 us forward and 92 backward, 990 in twos 70 and 129, 1023 as single elements 87 and 170.)
template <typename Rows> int widest(int most, int C, int Cg, Rows rows)
{
    int V = most;
    while (V > 1 && !(C % V == 0 && vectors_fit(Cg, V) && rows(V))) V /= 2;
    return V;
}

Cut cut_of(long long HW, int C, int G)
{
    Cut k = {};
    k.HW = HW; k.C = C; k.G = G; k.Cg = C / G; k.pieces = 1;
    return k;
}
// The rest of a cut, once its slab and tiles are chosen.
void finish_cut(Cut &k, int V)
{
    const int VW = k.slab / V, u = joined(k.Cg, V);
    k.rows = (k.HW + k.tiles - 1) / k.tiles;
    k.groups = std::max(1, k.slab / k.Cg);
    k.R = kGnThreads / VW;
    const long long pixels = (k.rows + k.R - 1) / k.R;
    k.head = pixels <= 8 ? 1 : pixels <= 32 ? 2 : 4;
    // lanes of a warp with the same channels: where their places are the same in every warp
    k.joint = VW <= 32 && 32 % VW == 0 ? 32 / VW : 1;
    k.least = 32 / k.joint;
    k.rows_of_sums = k.joint > 1 ? kGnThreads / 32 : k.R;
    k.per = std::min(k.slab, k.Cg) / u;
    k.sets = k.groups * k.per;
    k.lg_u = u == 8 ? 3 : u == 4 ? 2 : u == 2 ? 1 : 0;
    k.inv_n = 1.0 / ((double)k.HW * (double)k.Cg);
    // so that all groups have some at once, of a warp at most
    auto lanes = [&](int parts) {
        int lg = 0;
        while (lg < 5 && (1 << lg) < parts && (2 << lg) * k.groups <= kGnThreads) ++lg;
        return lg;
    };
    k.lg_tile = lanes(k.rows_of_sums * k.per);
    k.lg_slab = lanes(k.pieces * k.tiles);
    k.by_tiles = Div(k.tiles);
    k.by_slabs = Div(k.slabs);
    k.by_vectors = Div(VW);
    k.by_group = Div(k.Cg);
    k.by_per = Div(k.per);
}

// Slabs of a cluster: their data of `bytes` an element is resident in at most kMaxCluster blocks, beside beside(k) bytes of each.  False where they are not.
// Two blocks an SM, and slabs whose pixels have 64 bytes of all tensors together (at the time 64 x 12544 x 64 bf16 forward 53.6 us, with 32 bytes 64.2; 64 x 3136 x 256
// backward 112 us with 32 of each tensor, 122 with 64); of 32 bytes of a tensor where that alone gives the SMs a block each, or leaves no more than a cluster holds; where only the
// first are held they stay.  Of small images a block has more channels, up to 64 KB, as long as there is a block for each SM (64 x 49 x 512 bf16 5.0 us for 14.0, its
// backward pass 9.1 for 26.8; with a half of that least 64 x 784 x 512 took 34 us for 29, with twice as much its backward pass 75 for 55).  Smaller tiles, three or
// four blocks an SM, took longer: what a block does beside its elements is half of its instructions.
template <typename Beside> bool cut_resident(Cut &k, long long B, int V, int least_size, int bytes, Beside beside, size_t *smem)
{
    const int unit = (int)std::lcm((long long)k.Cg, (long long)V), units = k.C / unit;
    if (unit / V > kGnThreads) return false;
    auto need = [&](int tiles) {
        k.tiles = tiles;
        finish_cut(k, V);
        return (size_t)((k.rows + k.R - 1) / k.R) * kGnThreads * V * bytes + (beside(k) + 15) / 16 * 16;
    };
    auto tiles_for = [&](size_t most) {
        int tiles = 1;
        while (tiles <= kMaxCluster && need(tiles) > most) tiles *= 2;
        return tiles;
    };
    int tiles = kMaxCluster + 1, slab = 0;                           // tiles that a cluster holds, and their slab's channels
    for (const int channels : {64 / bytes, 32 / least_size}) {
        int of = std::max(1, std::min(units, channels / unit));
        while (units % of) --of;
        while (of < units && k.HW * unit * of * bytes < (long long)kTileLeast) {
            int more = of + 1;
            while (units % more) ++more;
            if (B * (units / more) < kSms || more * (unit / V) > kGnThreads || k.HW * unit * more * bytes > (long long)kTileTwo) break;
            of = more;
        }
        k.slab = unit * of;
        k.slabs = units / of;
        const int fit = tiles_for(kTileTwo);
        if (fit > kMaxCluster) continue;
        tiles = fit;
        slab = k.slab;
        while (B * k.slabs * tiles < kSms && tiles < kMaxCluster && k.HW * (k.slab / V) / (2 * tiles) >= 4 * kGnThreads) tiles *= 2;
        if (B * k.slabs * tiles >= kSms) break;
    }
    if (slab) {
        k.slab = slab;
        k.slabs = k.C / slab;
    } else {
        tiles = tiles_for(kTileMost);
    }
    if (tiles > kMaxCluster) return false;
    *smem = need(tiles);
    return B * k.slabs * k.tiles < 1ll << 31;
}
// Slabs and tiles of the two launches.
bool cut_streamed(Cut &k, long long B, int V)
{
    const long long unit = std::lcm((long long)k.Cg, (long long)V);
    k.pieces = 1;
    if (unit / V <= kGnThreads) {
        // whole groups: about 32 vectors a pixel
        const int units = (int)(k.C / unit);
        int of = (int)std::max(1ll, std::min<long long>(units, 32 * V / unit));
        while (units % of) --of;
        k.slab = (int)unit * of;
        k.slabs = units / of;
    } else {
        k.slab = kGnThreads * V;
        k.pieces = (k.Cg + k.slab - 1) / k.slab;
        k.slabs = k.G * k.pieces;
    }
    // about eight blocks an SM, of eight pixels a thread at least, and as many as there may be: where an image has many groups a slab,
    // few images of them are fewer blocks than SMs (128 of one image of 32 groups)
    const int R = std::max(1, kGnThreads / (k.slab / V));
    const long long want = std::max(1ll, 8ll * kSms / (B * k.slabs)), most = std::max(1ll, k.HW / (8ll * R));
    // (their sums are read by every block: sixteen of a thread at most, or 64 tiles; not measured against more)
    const long long read = std::max(64ll, 16ll * kGnThreads / (std::max(1, k.slab / k.Cg) * k.pieces));
    k.tiles = (int)std::min(read, std::min(want, most));
    finish_cut(k, V);
    return B * k.slabs * k.tiles < 1ll << 31 && k.rows < 1ll << 31;
}

// How a call of vectors of V elements is cut, `bytes` an element of all that it keeps and `least` of the smallest.  TWN_OK or why not.
struct Plan {
    bool resident;
    size_t smem;
};
template <typename Beside> int plan(Cut &k, Plan &p, long long B, int V, int least, int bytes, Beside beside)
{
    p.resident = cut_resident(k, B, V, least, bytes, beside, &p.smem);
    return p.resident || cut_streamed(k, B, V) ? TWN_OK : TWN_ERR_TOO_LARGE;
}
// Tiles that a workspace has room for: those of the call, and those of any batch of fewer images, which may have more tiles each.
long long tiles_at_most(const Cut &k, long long B, int V, bool resident)
{
    Cut one = k;
    if (!resident) cut_streamed(one, 1, V);
    return std::max(B * k.tiles, resident ? std::min<long long>(B * kMaxCluster, 2 * kSms) : std::min<long long>(B * one.tiles, 8 * kSms));
}

// That a block is there, and nothing about its memory: no write has to arrive before it.
__device__ __forceinline__ void arrive_first() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
// (threads of a warp that have gone different ways come together before its barrier)
__device__ __forceinline__ void arrive()
{
    __syncwarp();
    cluster_arrive();
}
__device__ __forceinline__ void wait_for_all()
{
    __syncwarp();
    cluster_wait();
}

// A grid of clusters of `cluster` blocks that may start while the kernel before it drains.
template <typename... KArgs, typename... Args>
cudaError_t launch_clusters(void (*kernel)(KArgs...), long long grid, int cluster, size_t smem, cudaStream_t s, const Args &...args)
{
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kGnThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}
template <typename Kernel> int allow_tile(Kernel kernel, int device, bool (&done)[64])
{
    if (!done[device]) TWN_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kTileMost));
    done[device] = true;
    return TWN_OK;
}

// B images of HW pixels of C channels in G groups: TWN_OK or why not.
int check_groups(long long B, long long HW, long long C, int G)
{
    TWN_REQUIRE(B >= 0 && HW >= 0 && C >= 1 && C <= 1 << 20 && G >= 1 && C % G == 0, TWN_ERR_INVALID_ARG);
    TWN_REQUIRE(B <= 1ll << 31 && HW <= 1ll << 31 && (B == 0 || HW <= (1ll << 40) / B), TWN_ERR_TOO_LARGE);
    return TWN_OK;
}

}  // namespace
