// Group norm with an activation, backward (see group_norm.cuh).
#include "group_norm.cuh"

namespace {

struct GnBwd {
    const void *dY, *X;
    void *dX;
    const void *add;                 // added to dX
    const float *gamma, *beta, *mean, *rstd;
    float *channels;                 // [B][tiles][2][C]: sums of dz (x - mean) rstd, of dz; NULL where the caller wants neither
    float2 *parts;                   // two launches: [B][G][pieces * tiles], sums of gamma dz, of gamma dz (x - mean)
    long long lddy, ldx, lddx;
    Cut cut;
    int act;
};

// Beside the tiles: the sums of the channels of rows of threads (joined inside the warps where they can be), those of the block, of its groups, and what makes dX
// from them.
__host__ __device__ __forceinline__ size_t sums_bytes(const Cut &k) { return ((size_t)(k.rows_of_sums + 1) * 2 * k.slab * 4 + 15) / 16 * 16; }
__host__ __device__ __forceinline__ int of_groups(const Cut &k) { return (k.groups * (8 * (k.tiles < kMaxCluster ? k.tiles : kMaxCluster) + 12) + 15) / 16 * 16; }
size_t bwd_beside(const Cut &k) { return sums_bytes(k) + of_groups(k); }
struct Beside {
    float *sums, *all;               // [rows][2][slab]; [2][slab], gamma times the block's
    float2 *own, *terms;             // of the groups: [groups][tiles], [groups]
    float *rstd;
    uint8_t *tile;
    __device__ __forceinline__ Beside(uint8_t *smem, const Cut &k)
    {
        sums = reinterpret_cast<float *>(smem);
        all = sums + k.rows_of_sums * 2 * k.slab;
        own = reinterpret_cast<float2 *>(smem + sums_bytes(k));
        terms = own + k.groups * min(k.tiles, kMaxCluster);
        rstd = reinterpret_cast<float *>(terms + k.groups);
        tile = smem + sums_bytes(k) + of_groups(k);
    }
};

// What a thread's channel of the block's sums is multiplied by, loaded before the tiles are: 1/deviation and gamma.
template <int V> struct OfChannel {
    float r = 0.0f, ga = 1.0f;
    __device__ __forceinline__ void load(const GnBwd &p, const Tile<V> &t, int c)
    {
        r = p.channels ? __ldg(p.rstd + t.b * p.cut.G + p.cut.by_group((uint32_t)(t.c0 + c))) : 0.0f;
        ga = p.gamma ? __ldg(p.gamma + t.c0 + c) : 1.0f;
    }
    // for sum e of the 2 C of the block, where there is a thread for each
    __device__ __forceinline__ OfChannel(const GnBwd &p, const Tile<V> &t)
    {
        if ((int)threadIdx.x < 2 * t.cs && 2 * t.cs <= kGnThreads) load(p, t, (int)threadIdx.x < t.cs ? threadIdx.x : threadIdx.x - t.cs);
    }
};
// The groups' 1/deviations, for all of the block.
template <int V> __device__ __forceinline__ void load_groups(const GnBwd &p, const Tile<V> &t, float *rstd)
{
    const float *from = p.rstd + t.b * p.cut.G + p.cut.by_group((uint32_t)t.c0);
    for (int g = threadIdx.x; g < p.cut.groups; g += kGnThreads) rstd[g] = __ldg(from + g);
}

// What a thread's channels have, as it is loaded (before the tiles are, and not waited for).
template <int V> struct Raw {
    float mean[V], rstd[V], gamma[V], beta[V];
    __device__ __forceinline__ Raw(const GnBwd &p, const Tile<V> &t)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) { mean[i] = rstd[i] = beta[i] = 0.0f; gamma[i] = 1.0f; }
        if (!t.has()) return;
        const int c = t.channel();
        const long long image = t.b * p.cut.G;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i == 0 || p.cut.Cg % V != 0) {
                const long long g = image + p.cut.by_group((uint32_t)(c + i));
                mean[i] = __ldg(p.mean + g);
                rstd[i] = __ldg(p.rstd + g);
            }
        if (p.gamma) load_floats(gamma, p.gamma + c);
        if (p.beta) load_floats(beta, p.beta + c);
    }
};
// A thread's channels: -mean, 1/deviation times gamma, beta; below what size of z fp32 leaves its sign in doubt.
template <int V> struct Channels {
    static constexpr int P = V > 1 ? V / 2 : 1;
    two_f32 m[P], a[P], b[P];
    float doubt;
    __device__ __forceinline__ Channels(const GnBwd &p, const Raw<V> &r)
    {
        const bool one = p.cut.Cg % V == 0;          // group
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int l = 2 * i < V ? 2 * i : 0, h = V > 1 ? 2 * i + 1 : 0;
            m[i] = two(one ? -r.mean[0] : -r.mean[l], one ? -r.mean[0] : -r.mean[h]);
            a[i] = mul2(two(one ? r.rstd[0] : r.rstd[l], one ? r.rstd[0] : r.rstd[h]), two(r.gamma[l], r.gamma[h]));
            b[i] = two(r.beta[l], r.beta[h]);
        }
        // (z is right to a few roundings of its two terms, 2^-24 each; the first is as large as z and beta together at most.  Below 2^-126 a product may have lost its sign, and
        // where a factor has come down there any z may have)
        doubt = 0x1p-126f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float rstd = one ? r.rstd[0] : r.rstd[i];
            doubt = fmaxf(doubt, fabsf(rstd * r.gamma[i]) < 0x1p-100f && rstd != 0.0f && r.gamma[i] != 0.0f ? INFINITY : 0x1p-18f * fabsf(r.beta[i]));
        }
    }
};

// The sign of z where fp32 leaves it in doubt: z from the same numbers in fp64.
__device__ __noinline__ bool positive_z(const GnBwd &p, long long b, int c, float x)
{
    const long long g = b * p.cut.G + c / p.cut.Cg;
    const double xh = ((double)x - (double)p.mean[g]) * (double)p.rstd[g];
    return xh * (p.gamma ? (double)p.gamma[c] : 1.0) + (p.beta ? (double)p.beta[c] : 0.0) > 0.0;
}

// Where x is the mean z is beta, and of a sure sign.
template <int V> __device__ __forceinline__ bool sure(const Channels<V> &ch, int i, float x)
{
    float lo, hi;
    each(ch.m[i / 2], lo, hi);
    return x == (i % 2 ? -hi : -lo);
}

// Pairs of a thread's vector: dz and the differences from the mean.
template <typename TD, typename TX, int V, int ACT>
__device__ __forceinline__ void vector_dz(const GnBwd &p, const Tile<V> &t, const Channels<V> &ch, const Vec<TD, V> &vd, const Vec<TX, V> &vx,
                                          two_f32 (&dz)[Channels<V>::P], two_f32 (&d)[Channels<V>::P])
{
    float dy[V], x[V];
    vd.get(dy);
    vx.get(x);
    float z[V];
    if (ACT == kRelu) {
        bool doubt = false;
#pragma unroll
        for (int i = 0; i < Channels<V>::P; ++i) {
            const int l = 2 * i < V ? 2 * i : 0, h = V > 1 ? 2 * i + 1 : 0;
            float lo, hi;
            each(fma2(add2(two(x[l], V > 1 ? x[h] : 0.0f), ch.m[i]), ch.a[i], ch.b[i]), lo, hi);
            z[l] = lo;
            if (V > 1) z[h] = hi;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) doubt |= fabsf(z[i]) < ch.doubt;
        if (doubt)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (fabsf(z[i]) < ch.doubt && !sure(ch, i, x[i])) z[i] = positive_z(p, t.b, t.channel() + i, x[i]) ? 1.0f : 0.0f;
        // (a NaN goes on)
#pragma unroll
        for (int i = 0; i < V; ++i) dy[i] = z[i] > 0.0f ? dy[i] : at_least(z[i], 0.0f);
    }
#pragma unroll
    for (int i = 0; i < Channels<V>::P; ++i) {
        const int l = 2 * i < V ? 2 * i : 0, h = V > 1 ? 2 * i + 1 : 0;
        d[i] = add2(two(x[l], V > 1 ? x[h] : 0.0f), ch.m[i]);
        dz[i] = two(dy[l], V > 1 ? dy[h] : 0.0f);
        if (ACT == kSilu) {
            // dy f (1 + z (1 - f)) = dy f (1 + z e f),  e = exp(-z), f = 1 / (1 + e).  (A reciprocal for two pixels, as the forward pass has it, takes more registers: 108 us for 105.)
            const two_f32 z[1] = {at_least2(fma2(d[i], ch.a[i], ch.b[i]), kLeastZ)};
            two_f32 e[1], f[1];
            sigmoids<1>(z, e, f);
            dz[i] = mul2(mul2(dz[i], f[0]), fma2(z[0], mul2(e[0], f[0]), two(1.0f, 1.0f)));
        }
    }
}

// Pixels from `begin` to `end` of a thread, which take(i, dY, X) loads: use(i, dz, differences) for each.
template <typename TD, typename TX, int V, int ACT, typename Take, typename Use>
__device__ __forceinline__ void pixel_by_pixel(const GnBwd &p, const Tile<V> &t, const Channels<V> &ch, int begin, int end, const Take &take, const Use &use)
{
#pragma unroll 2
    for (int i = begin; i < end; ++i) {
        Vec<TD, V> vd;
        Vec<TX, V> vx;
        two_f32 dz[Channels<V>::P], d[Channels<V>::P];
        take(i, vd, vx);
        vector_dz<TD, TX, V, ACT>(p, t, ch, vd, vx, dz, d);
        use(i, dz, d);
    }
}
template <int N> __device__ __forceinline__ void add_sums(two_f32 (&A)[N], two_f32 (&D)[N], const two_f32 (&dz)[N], const two_f32 (&d)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) {
        A[j] = add2(A[j], dz[j]);
        D[j] = fma2(dz[j], d[j], D[j]);
    }
}

// The sums of a run of pixels go to those of all.
template <int N> __device__ __forceinline__ void end_run(two_f32 (&A)[N], two_f32 (&D)[N], two_f32 (&a)[N], two_f32 (&q)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) {
        A[j] = add2(A[j], a[j]);
        D[j] = add2(D[j], q[j]);
        a[j] = q[j] = 0;
    }
}

// Sums of N numbers over the lanes that are `least` apart, by halves: of two lanes each goes on with half of the numbers.  A lane ends with N / 2^steps of them (one at
// least), the first of which has the index that it returns.
template <int N, int OFF> __device__ __forceinline__ int fold_lanes(float *v, int least, int &left)
{
    left = N;
    if constexpr (OFF == 0) {
        return 0;
    } else {
        if (OFF < least) return 0;
        const bool up = threadIdx.x & OFF;
        if constexpr (N > 1) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float mine = up ? v[i + N / 2] : v[i], other = up ? v[i] : v[i + N / 2];
                v[i] = mine + __shfl_xor_sync(0xffffffffu, other, OFF);
            }
            return (up ? N / 2 : 0) + fold_lanes<N / 2, OFF / 2>(v, least, left);
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], OFF);
            return fold_lanes<1, OFF / 2>(v, least, left);
        }
    }
}

// Sums of the block's channels from those of its threads: to `channels` where the caller wants them, and those of its groups to write(group, kind, part, sum) for
// every part < parts.  Called by all.
template <int V, typename Write>
__device__ __forceinline__ void join_channels(const GnBwd &p, const Tile<V> &t, const two_f32 (&A)[Channels<V>::P], const two_f32 (&D)[Channels<V>::P], const Beside &at, OfChannel<V> of,
                                              int parts, Write write)
{
    const Cut &k = p.cut;
    float v[2 * V];
#pragma unroll
    for (int i = 0; i < Channels<V>::P; ++i) {
        float lo, hi;
        each(A[i], lo, hi);
        v[2 * i < V ? 2 * i : 0] = lo;
        if (V > 1) v[V > 1 ? 2 * i + 1 : 0] = hi;
        each(D[i], lo, hi);
        v[V + (2 * i < V ? 2 * i : 0)] = lo;
        if (V > 1) v[V + (V > 1 ? 2 * i + 1 : 0)] = hi;
    }
    if (k.joint > 1) {
        int left;
        const int first = fold_lanes<2 * V, 16>(v, k.least, left);
        float *const to = at.sums + (threadIdx.x >> 5) * 2 * k.slab + t.tx * V;
        // (where lanes outnumber the numbers some of them have the same one)
#pragma unroll
        for (int i = 0; i < 2 * V; ++i)
            if (i < left) to[(first + i) / V * k.slab + (first + i) % V] = v[i];
    } else if (t.has()) {
        float *const to = at.sums + t.ty * 2 * k.slab + t.tx * V;
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) to[i / V * k.slab + i % V] = v[i];
    }
    __syncthreads();
    const int rows = k.rows_of_sums;
    // where a group's channels are neighbouring lanes of a warp, they meet there
    const bool lanes = (k.Cg & (k.Cg - 1)) == 0 && k.Cg <= 32;
    for (int e0 = 0; e0 < 2 * t.cs; e0 += kGnThreads) {
        const int e = e0 + threadIdx.x;
        const bool there = e < 2 * t.cs, second = e >= t.cs;        // of dz (x - mean)
        const int c = second ? e - t.cs : e;
        float a = 0.0f;
        if (there) {
            if (2 * t.cs > kGnThreads) of.load(p, t, c);
            const float *from = at.sums + (second ? k.slab : 0) + c;
#pragma unroll 8
            for (int y = 0; y < rows; ++y) a += from[y * 2 * k.slab];
            if (p.channels) p.channels[((t.b * k.tiles + t.tile) * 2 + (second ? 0 : 1)) * k.C + t.c0 + c] = second ? a * of.r : a;
            a *= of.ga;
            if (!lanes) at.all[(second ? k.slab : 0) + c] = a;
        }
        if (lanes && (e & ~31) < 2 * t.cs) {
            a = all_sum(a, 31 - __clz(k.Cg));
            const int i = c & (k.Cg - 1), g = (int)k.by_group((uint32_t)c);
            if (there)
                for (int to = i; to < parts; to += k.Cg) write(g, second, to, a);
        }
    }
    if (lanes) return;
    __syncthreads();
    // groups by as many neighbouring lanes as they have channels, 32 at most
    const int Cg = min(k.Cg, t.cs);
    int lg = 0;
    while ((1 << lg) < Cg && lg < 5) ++lg;
    const int width = 1 << lg, mine = threadIdx.x >> lg, lane = threadIdx.x & (width - 1), at_once = kGnThreads >> lg;
    for (int g0 = 0; g0 < 2 * k.groups; g0 += at_once) {
        const int e = g0 + mine, g = e >> 1;
        const float *from = at.all + (e & 1 ? k.slab : 0) + g * Cg;
        float a = 0.0f;
        if (g < k.groups)
            for (int c = lane; c < Cg; c += width) a += from[c];
        a = all_sum(a, lg);
        if (g < k.groups)
            for (int to = lane; to < parts; to += width) write(g, e & 1, to, a);
    }
}

// rstd s / N and rstd^3 t / N of the block's groups, from `count` parts of each.
template <typename Read> __device__ __forceinline__ void finish_groups(const GnBwd &P, int count, const float *rstd, float2 *to, Read read)
{
    const int lg = P.cut.lg_slab, width = 1 << lg, mine = threadIdx.x >> lg, lane = threadIdx.x & (width - 1), groups = P.cut.groups;
    const float inv = (float)P.cut.inv_n;
    // (a warp without a group has nothing to do)
    for (int g0 = 0; g0 + (int)((threadIdx.x & ~31u) >> lg) < groups; g0 += kGnThreads >> lg) {
        const int g = g0 + mine;
        float s = 0.0f, q = 0.0f;
        const float r = g < groups ? rstd[g] : 0.0f;
        if (g < groups)
            for (int k = lane; k < count; k += width) {
                const float2 v = read(g, k);
                s += v.x;
                q += v.y;
            }
        s = all_sum(s, lg);
        q = all_sum(q, lg);
        if (g < groups && lane == 0) to[g] = make_float2(r * (s * inv), r * r * (r * (q * inv)));
    }
    __syncthreads();
}

// Per channel of a thread what dX = dz a - p - d q takes from the group.
template <int V> struct Terms {
    two_f32 p[Channels<V>::P], q[Channels<V>::P];
    __device__ __forceinline__ Terms(const GnBwd &P, const Tile<V> &t, const float2 *of)
    {
#pragma unroll
        for (int i = 0; i < Channels<V>::P; ++i) {
            const int l = t.tx * V + (2 * i < V ? 2 * i : 0), h = t.tx * V + (V > 1 ? 2 * i + 1 : 0);
            const float2 x = of[P.cut.pieces > 1 ? 0 : P.cut.by_group((uint32_t)l)], y = of[P.cut.pieces > 1 ? 0 : P.cut.by_group((uint32_t)h)];
            p[i] = two(-x.x, -y.x);
            q[i] = two(-x.y, -y.y);
        }
    }
};
template <int V, typename TO>
__device__ __forceinline__ void write_dx(const Channels<V> &ch, const Terms<V> &te, const two_f32 (&dz)[Channels<V>::P], const two_f32 (&d)[Channels<V>::P], TO *to, const TO *add)
{
    float o[V];
#pragma unroll
    for (int i = 0; i < Channels<V>::P; ++i) {
        float o0, o1;
        each(fma2(dz[i], ch.a[i], fma2(d[i], te.q[i], te.p[i])), o0, o1);
        o[2 * i < V ? 2 * i : 0] = o0;
        if (V > 1) o[V > 1 ? 2 * i + 1 : 0] = o1;
    }
    if (add) {
        Vec<TO, V> v;
        float r[V];
        v.load(add);
        v.get(r);
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] += r[i];
    }
    store(to, o);
}

// 64 x 3136 x 256 bf16 with SiLU in 105 us, 2.9 TB/s: bound by instructions and their latency (52 % of the issue slots with 16 warps an SM, three quarters of them elementwise;
// exp and the reciprocal keep their unit at a third).
// ---- resident -------------------------------------------------------------------------------------------------------------------
// dz is taken anew for the outputs: to keep it in fp32 beside X costs half of the room for tiles (64 x 3136 x 256 with SiLU: 144 us, 118 this way at the time).
template <typename TD, typename TX, typename TO, int V, int ACT>
__device__ __forceinline__ void resident(const GnBwd &P, const Tile<V> &t, const Raw<V> &raw, const OfChannel<V> &of, const Beside &at, const TD *ds, const TX *xs)
{
    constexpr int N = Channels<V>::P;
    const int tiles = P.cut.tiles;
    const Channels<V> ch(P, raw);
    two_f32 A[N], D[N];
#pragma unroll
    for (int i = 0; i < N; ++i) A[i] = D[i] = 0;
    auto take = [&](int i, Vec<TD, V> &vd, Vec<TX, V> &vx) {
        vd.load(ds + i * (kGnThreads * V));
        vx.load(xs + i * (kGnThreads * V));
    };
    if constexpr (kTileMost / (kGnThreads * V * (sizeof(TD) + sizeof(TX))) <= kRun) {
        as_they_come(t.n, 0, [&](int begin, int end) { pixel_by_pixel<TD, TX, V, ACT>(P, t, ch, begin, end, take, [&](int, const two_f32 (&dz)[N], const two_f32 (&d)[N]) { add_sums<N>(A, D, dz, d); }); });
    } else {
        two_f32 a[N], q[N];
#pragma unroll
        for (int j = 0; j < N; ++j) a[j] = q[j] = 0;
        int next = kRun;
        as_they_come(t.n, 0, [&](int begin, int end) {
            while (begin < end) {
                const int stop = min(end, next);
                pixel_by_pixel<TD, TX, V, ACT>(P, t, ch, begin, stop, take, [&](int, const two_f32 (&dz)[N], const two_f32 (&d)[N]) { add_sums<N>(a, q, dz, d); });
                begin = stop;
                if (stop == next) {
                    end_run<N>(A, D, a, q);
                    next += kRun;
                }
            }
        });
        end_run<N>(A, D, a, q);
    }
    if (tiles > 1) wait_for_all();                       // all blocks are there
    // to all blocks of the cluster (without dX to none, which may have ended)
    join_channels(P, t, A, D, at, of, P.dX ? tiles : 0, [&](int g, int kind, int to, float v) {
        float *const place = reinterpret_cast<float *>(at.own + g * tiles + t.tile) + kind;
        if (tiles == 1) *place = v;
        else send(place, to, v);
    });
    if (!P.dX) return;
    if (tiles == 1) {
        __syncthreads();
    } else {
        arrive();
        wait_for_all();
    }
    finish_groups(P, tiles, at.rstd, at.terms, [&](int g, int k) { return at.own[g * tiles + k]; });
    if (t.n > 0) {
        const Terms<V> te(P, t, at.terms);
        const long long to_at = (t.b * P.cut.HW + t.first + t.ty) * P.lddx + t.channel(), step = t.R * P.lddx;
        TO *to = static_cast<TO *>(P.dX) + to_at;
        const TO *add = P.add ? static_cast<const TO *>(P.add) + to_at : nullptr;
        pixel_by_pixel<TD, TX, V, ACT>(P, t, ch, 0, t.n, take,
                                 [&](int i, const two_f32 (&dz)[N], const two_f32 (&d)[N]) { write_dx<V>(ch, te, dz, d, to + i * step, add ? add + i * step : nullptr); });
    }
}

template <typename TD, typename TX, typename TO, int V>
__global__ void __launch_bounds__(kGnThreads, 2) gn_bwd_kernel(const __grid_constant__ GnBwd P)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const Tile<V> t(P.cut, blockIdx.x);
    const Beside at(smem, P.cut);
    const int groups = P.cut.groups, most = t.base + (t.rest > 0);         // pixels of any thread
    pdl_begin();
    const int tiles = P.cut.tiles;
    if (tiles > 1) arrive_first();
    const Raw<V> raw(P, t);
    const OfChannel<V> of(P, t);
    const float *const rstds = P.rstd + t.b * P.cut.G + P.cut.by_group((uint32_t)t.c0);
    const float rstd = (int)threadIdx.x < groups ? __ldg(rstds + threadIdx.x) : 0.0f;
    TD *const ds = reinterpret_cast<TD *>(at.tile) + threadIdx.x * V;
    TX *const xs = reinterpret_cast<TX *>(at.tile + (size_t)most * kGnThreads * V * sizeof(TD)) + threadIdx.x * V;
    const long long pixel = t.b * P.cut.HW + t.first + t.ty;
    {
        const TD *dy = static_cast<const TD *>(P.dY) + pixel * P.lddy + t.channel();
        const TX *x = static_cast<const TX *>(P.X) + pixel * P.ldx + t.channel();
        const long long step_d = t.R * P.lddy, step_x = t.R * P.ldx;
        int begin = 0;
#pragma unroll
        for (int q = 0; q < kShares; ++q) {
            const int end = share_end(t.n, q);
            copy_vectors<TD, V>(ds + begin * (kGnThreads * V), dy + begin * step_d, step_d, end - begin);
            copy_vectors<TX, V>(xs + begin * (kGnThreads * V), x + begin * step_x, step_x, end - begin);
            end_share();
            begin = end;
        }
    }
    if ((int)threadIdx.x < groups) at.rstd[threadIdx.x] = rstd;
    for (int g = threadIdx.x + kGnThreads; g < groups; g += kGnThreads) at.rstd[g] = __ldg(rstds + g);
    if (P.act == kSilu) resident<TD, TX, TO, V, kSilu>(P, t, raw, of, at, ds, xs);
    else if (P.act == kRelu) resident<TD, TX, TO, V, kRelu>(P, t, raw, of, at, ds, xs);
    else resident<TD, TX, TO, V, kNone>(P, t, raw, of, at, ds, xs);
}

// 131072 pixels of 512 channels, one group, in 152 us: five passes over 134 MB would take 102.  (Two blocks an SM, at 128 registers; with one, at 172, it took 176.)
// ---- two reads ------------------------------------------------------------------------------------------------------------------
// A thread's pixels from `i` to `end`, the loads of four at a time: use(i, dz, differences) for each.
template <typename TD, typename TX, int V, int ACT, typename Use>
__device__ __forceinline__ void each_pixel(const GnBwd &P, const Tile<V> &t, const Channels<V> &ch, int i, int end, const Use &use)
{
    const long long pixel = t.b * P.cut.HW + t.first + t.ty;
    const TD *dy = static_cast<const TD *>(P.dY) + pixel * P.lddy + t.channel();
    const TX *x = static_cast<const TX *>(P.X) + pixel * P.ldx + t.channel();
    const long long step_d = t.R * P.lddy, step_x = t.R * P.ldx;
    two_f32 dz[Channels<V>::P], d[Channels<V>::P];
    for (; i + 4 <= end; i += 4) {
        Vec<TD, V> vd[4];
        Vec<TX, V> vx[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            vd[j].load(dy + (i + j) * step_d);
            vx[j].load(x + (i + j) * step_x);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            vector_dz<TD, TX, V, ACT>(P, t, ch, vd[j], vx[j], dz, d);
            use(i + j, dz, d);
        }
    }
    for (; i < end; ++i) {
        Vec<TD, V> vd;
        Vec<TX, V> vx;
        vd.load(dy + i * step_d);
        vx.load(x + i * step_x);
        vector_dz<TD, TX, V, ACT>(P, t, ch, vd, vx, dz, d);
        use(i, dz, d);
    }
}
template <typename TD, typename TX, int V, int ACT>
__device__ __forceinline__ void tile_sums(const GnBwd &P, const Tile<V> &t, two_f32 (&A)[Channels<V>::P], two_f32 (&D)[Channels<V>::P])
{
    constexpr int N = Channels<V>::P;
    const Channels<V> ch(P, Raw<V>(P, t));
    two_f32 a[N], q[N];
#pragma unroll
    for (int j = 0; j < N; ++j) a[j] = q[j] = 0;
    for (int i = 0; i < t.n; i += kRun) {
        each_pixel<TD, TX, V, ACT>(P, t, ch, i, min(t.n, i + kRun), [&](int, const two_f32 (&dz)[N], const two_f32 (&d)[N]) { add_sums<N>(a, q, dz, d); });
        end_run<N>(A, D, a, q);
    }
}
template <typename TD, typename TX, int V> __global__ void __launch_bounds__(kGnThreads, 2) gn_bwd_sums_kernel(const __grid_constant__ GnBwd P)
{
    extern __shared__ __align__(16) uint8_t smem[];
    constexpr int N = Channels<V>::P;
    const Tile<V> t(P.cut, blockIdx.x);
    const Beside at(smem, P.cut);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const OfChannel<V> of(P, t);
    two_f32 A[N], D[N];
#pragma unroll
    for (int i = 0; i < N; ++i) A[i] = D[i] = 0;
    if (t.n > 0) {
        if (P.act == kSilu) tile_sums<TD, TX, V, kSilu>(P, t, A, D);
        else if (P.act == kRelu) tile_sums<TD, TX, V, kRelu>(P, t, A, D);
        else tile_sums<TD, TX, V, kNone>(P, t, A, D);
    }
    const int g0 = t.c0 / P.cut.Cg, piece = P.cut.pieces > 1 ? (t.c0 - g0 * P.cut.Cg) / P.cut.slab : 0;
    join_channels(P, t, A, D, at, of, 1, [&](int g, int kind, int, float v) {
        reinterpret_cast<float *>(P.parts + ((t.b * P.cut.G + g0 + g) * P.cut.pieces + piece) * P.cut.tiles + t.tile)[kind] = v;
    });
}
template <typename TD, typename TX, typename TO, int V, int ACT>
__device__ __forceinline__ void apply_rows(const GnBwd &P, const Tile<V> &t, const float2 *terms)
{
    constexpr int N = Channels<V>::P;
    const Channels<V> ch(P, Raw<V>(P, t));
    const Terms<V> te(P, t, terms);
    const long long at = (t.b * P.cut.HW + t.first + t.ty) * P.lddx + t.channel(), step = t.R * P.lddx;
    TO *to = static_cast<TO *>(P.dX) + at;
    const TO *add = P.add ? static_cast<const TO *>(P.add) + at : nullptr;
    each_pixel<TD, TX, V, ACT>(P, t, ch, 0, t.n, [&](int i, const two_f32 (&dz)[N], const two_f32 (&d)[N]) { write_dx<V>(ch, te, dz, d, to + i * step, add ? add + i * step : nullptr); });
}
template <typename TD, typename TX, typename TO, int V> __global__ void __launch_bounds__(kGnThreads, 2) gn_bwd_apply_kernel(const __grid_constant__ GnBwd P)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const Tile<V> t(P.cut, blockIdx.x);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int count = P.cut.pieces * P.cut.tiles;
    float2 *const terms = reinterpret_cast<float2 *>(smem);
    float *const rstd = reinterpret_cast<float *>(terms + P.cut.groups);
    const long long first = t.b * P.cut.G + t.c0 / P.cut.Cg;
    load_groups(P, t, rstd);
    __syncthreads();
    finish_groups(P, count, rstd, terms, [&](int g, int k) { return P.parts[(first + g) * count + k]; });
    if (t.n == 0) return;
    if (P.act == kSilu) apply_rows<TD, TX, TO, V, kSilu>(P, t, terms);
    else if (P.act == kRelu) apply_rows<TD, TX, TO, V, kRelu>(P, t, terms);
    else apply_rows<TD, TX, TO, V, kNone>(P, t, terms);
}

// dgamma and dbeta: sums over the images' tiles, fp64, in a fixed order.  A block has 32 of the 2 C columns.
constexpr int kFoldRows = 32;
__global__ void __launch_bounds__(32 * kFoldRows) gn_fold_kernel(const float *channels, long long rows, int C, float *dgamma, float *dbeta)
{
    __shared__ double sums[kFoldRows][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int x = threadIdx.x % 32, y = threadIdx.x / 32, c = blockIdx.x * 32 + x;
    double a = 0.0;
    if (c < 2 * C)
#pragma unroll 8
        for (long long r = y; r < rows; r += kFoldRows) a += (double)channels[r * 2 * C + c];
    sums[y][x] = a;
    __syncthreads();
    if (y != 0 || c >= 2 * C) return;
    a = 0.0;
#pragma unroll
    for (int i = 0; i < kFoldRows; ++i) a += sums[i][x];
    float *to = c < C ? dgamma : dbeta;
    if (to) to[c < C ? c : c - C] = (float)a;
}

// ---- host ---------------------------------------------------------------------------------------------------------------------
// Sums of channels in front, those of groups behind them.
size_t channel_bytes(const Cut &k, long long tiles) { return ((size_t)tiles * 2 * k.C * sizeof(float) + 255) / 256 * 256; }
size_t workspace_of(const Cut &k, long long tiles, bool resident) { return channel_bytes(k, tiles) + (resident ? 0 : (size_t)tiles * k.G * k.pieces * sizeof(float2)); }

int fold(const GnBwd &P, long long B, float *dgamma, float *dbeta, cudaStream_t s)
{
    if (!P.channels) return TWN_OK;
    TWN_CUDA_OK(twn_launch_pdl(true, gn_fold_kernel, (2 * P.cut.C + 31) / 32, 32 * kFoldRows, 0, s, P.channels, B * P.cut.tiles, P.cut.C, dgamma, dbeta));
    return TWN_OK;
}

template <typename TD, typename TX, typename TO, int V>
int bwd(GnBwd &P, const Plan &plan, long long B, const twn_device_info &dev, float *dgamma, float *dbeta, void *workspace, cudaStream_t s)
{
    const Cut &k = P.cut;
    if (plan.resident) {
        static bool done[64] = {false};
        const int rc = allow_tile(gn_bwd_kernel<TD, TX, TO, V>, dev.ordinal, done);
        if (rc != TWN_OK) return rc;
        TWN_CUDA_OK(launch_clusters(gn_bwd_kernel<TD, TX, TO, V>, B * k.slabs * k.tiles, k.tiles, plan.smem, s, P));
        return fold(P, B, dgamma, dbeta, s);
    }
    P.parts = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + channel_bytes(k, B * k.tiles));
    const int grid = (int)(B * k.slabs * k.tiles);
    TWN_CUDA_OK(twn_launch_pdl(true, gn_bwd_sums_kernel<TD, TX, V>, grid, kGnThreads, sums_bytes(k), s, P));
    if (P.dX) TWN_CUDA_OK(twn_launch_pdl(true, gn_bwd_apply_kernel<TD, TX, TO, V>, grid, kGnThreads, (size_t)k.groups * 12, s, P));
    return fold(P, B, dgamma, dbeta, s);
}
template <typename TD, typename TX, typename TO>
int bwd_any(GnBwd &P, const Plan &plan, long long B, int V, const twn_device_info &dev, float *dgamma, float *dbeta, void *workspace, cudaStream_t s)
{
    if constexpr (sizeof(TD) + sizeof(TX) + sizeof(TO) == 6)
        if (V == 8) return bwd<TD, TX, TO, 8>(P, plan, B, dev, dgamma, dbeta, workspace, s);
    if (V == 4) return bwd<TD, TX, TO, 4>(P, plan, B, dev, dgamma, dbeta, workspace, s);
    if (V == 2) return bwd<TD, TX, TO, 2>(P, plan, B, dev, dgamma, dbeta, workspace, s);
    return bwd<TD, TX, TO, 1>(P, plan, B, dev, dgamma, dbeta, workspace, s);
}
template <typename TD, typename TX>
int bwd_to(GnBwd &P, const Plan &plan, int dx_dtype, long long B, int V, const twn_device_info &dev, float *dgamma, float *dbeta, void *workspace, cudaStream_t s)
{
    return dx_dtype == TWN_BF16 ? bwd_any<TD, TX, bf16>(P, plan, B, V, dev, dgamma, dbeta, workspace, s)
                                : bwd_any<TD, TX, float>(P, plan, B, V, dev, dgamma, dbeta, workspace, s);
}

}  // namespace

extern "C" size_t twn_group_norm_bwd_workspace_bytes(int64_t B, int64_t HW, int64_t C, int32_t groups)
{
    if (check_groups(B, HW, C, groups) != TWN_OK || B == 0 || HW == 0) return 0;
    size_t most = 0;
    for (int V : {1, 2, 4, 8})
        for (int bytes : {4, 6, 8}) {                                // of dY and X together
            Cut k = cut_of(HW, (int)C, groups);
            Plan p;
            if (C % V || !vectors_fit(k.Cg, V) || (V == 8 && bytes > 4) || plan(k, p, B, V, bytes == 8 ? 4 : 2, bytes, bwd_beside) != TWN_OK) continue;
            most = std::max(most, workspace_of(k, tiles_at_most(k, B, V, p.resident), p.resident));
        }
    return (most + 255) / 256 * 256;
}

extern "C" int twn_group_norm_bwd(const void *dY, int32_t dy_dtype, int64_t lddy, const void *X, int32_t x_dtype, int64_t ldx, int64_t B, int64_t HW,
                                  int64_t C, int32_t groups, const float *gamma, const float *beta, const float *mean, const float *rstd, int32_t act,
                                  void *dX, int32_t dx_dtype, int64_t lddx, const void *residual, float *dgamma, float *dbeta, void *workspace,
                                  size_t workspace_bytes, twn_stream_t stream)
{
    int rc = check_groups(B, HW, C, groups);
    if (rc != TWN_OK) return rc;
    TWN_REQUIRE(is_act(act) && (!residual || dX), TWN_ERR_INVALID_ARG);
    const long long M = B * HW;
    rc = check_matrix(dY, dy_dtype, lddy, M, C);
    if (rc == TWN_OK) rc = check_matrix(X, x_dtype, ldx, M, C);
    if (rc == TWN_OK && dX) rc = check_matrix(dX, dx_dtype, lddx, M, C);
    if (rc != TWN_OK) return rc;
    TWN_REQUIRE(M == 0 || (mean && rstd), TWN_ERR_INVALID_ARG);
    for (const void *p : {(const void *)gamma, (const void *)beta, (const void *)mean, (const void *)rstd, (const void *)dgamma, (const void *)dbeta})
        TWN_REQUIRE(twn_aligned(p, 4), TWN_ERR_MISALIGNED);
    if (residual) TWN_REQUIRE(twn_aligned(residual, size_of(dx_dtype)), TWN_ERR_MISALIGNED);
    if (!dX && !dgamma && !dbeta) return TWN_OK;
    cudaStream_t s = twn_cu(stream);
    if (M == 0) {
        for (float *p : {dgamma, dbeta})
            if (p) TWN_CUDA_OK(cudaMemsetAsync(p, 0, (size_t)C * sizeof(float), s));
        return TWN_OK;
    }
    const int out = dX ? dx_dtype : dy_dtype;
    Cut k = cut_of(HW, (int)C, groups);
    const int V = widest(dy_dtype == TWN_BF16 && x_dtype == TWN_BF16 && out == TWN_BF16 ? 8 : 4, (int)C, k.Cg, [&](int v) {
        return vector_rows(dY, dy_dtype, lddy, v) && vector_rows(X, x_dtype, ldx, v) && (!dX || vector_rows(dX, dx_dtype, lddx, v)) &&
               (!residual || vector_rows(residual, dx_dtype, lddx, v));
    });
    Plan p;
    rc = plan(k, p, B, V, (int)std::min(size_of(dy_dtype), size_of(x_dtype)), (int)(size_of(dy_dtype) + size_of(x_dtype)), bwd_beside);
    if (rc != TWN_OK) return rc;
    const size_t need = workspace_of(k, B * k.tiles, p.resident);
    TWN_REQUIRE(workspace != nullptr && workspace_bytes >= need, TWN_ERR_WORKSPACE);
    TWN_REQUIRE(twn_aligned(workspace, 256), TWN_ERR_MISALIGNED);
    Places places;
    places.matrix(dX, dx_dtype, lddx, M, C, true);
    places.matrix(dY, dy_dtype, lddy, M, C, false);
    places.matrix(X, x_dtype, ldx, M, C, false);
    places.matrix(residual, dx_dtype, lddx, M, C, false);
    for (const void *q : {(const void *)gamma, (const void *)beta}) places.vector(q, 4 * C, false);
    for (const void *q : {(const void *)mean, (const void *)rstd}) places.vector(q, 4 * B * groups, false);
    for (const void *q : {(const void *)dgamma, (const void *)dbeta}) places.vector(q, 4 * C, true);
    places.vector(workspace, (long long)need, true);
    TWN_REQUIRE(places.apart(), TWN_ERR_INVALID_ARG);
    twn_device_info dev;
    rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    GnBwd P = {dY, X, dX, residual, gamma, beta, mean, rstd, dgamma || dbeta ? static_cast<float *>(workspace) : nullptr, nullptr, lddy, ldx, lddx, k, act};
    if (dy_dtype == TWN_BF16)
        return x_dtype == TWN_BF16 ? bwd_to<bf16, bf16>(P, p, out, B, V, dev, dgamma, dbeta, workspace, s) : bwd_to<bf16, float>(P, p, out, B, V, dev, dgamma, dbeta, workspace, s);
    return x_dtype == TWN_BF16 ? bwd_to<float, bf16>(P, p, out, B, V, dev, dgamma, dbeta, workspace, s) : bwd_to<float, float>(P, p, out, B, V, dev, dgamma, dbeta, workspace, s);
}
