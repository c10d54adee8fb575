// Group norm with an activation, forward (see group_norm.cuh).
#include "group_norm.cuh"

#include <type_traits>

namespace {

// Of n values of a group: their mean as it is in fp32, their sum less n times that, the sum of squares of their differences from the mean.  Parts are joined by the differences of their
// means from one of those, which are no larger than what makes them differ: the group's mean keeps its digits however far from zero its values lie, and whichever of them is
// far from the others.  (Sums in fp64 keep as many and took more time, four conversions a part: 7 x 1023 x 132 fp32 in 7.9 us for 7.1.)
struct __align__(16) Moments {
    float c, r, m2, n;
};

struct GnFwd {
    const void *X;
    void *Y;
    const float *gamma, *beta;
    float *mean, *rstd;
    Moments *parts;                  // two launches: [B][G][pieces * tiles]
    long long ldx, ldy;
    Cut cut;
    int act;
    float eps;
};

// A group's values from their parts, which read(e) gives for e < count, in the 2^lg neighbouring lanes that call it (Chan, Golub and LeVeque): their sum and their mean less `c`, that of
// the first part, and the sum of squared differences.  inv: 1 / their number.
struct Joined {
    float c;
    double sum, mean;
    float m2;
};
template <typename Read> __device__ __forceinline__ Joined join(int lane, int lg, int count, double inv, Read read)
{
    const int width = 1 << lg;
    Moments held = {0.0f, 0.0f, 0.0f, 0.0f};             // the first of a lane's parts
    if (lane < count) held = read(lane);
    const float c = count > 0 ? read(0).c : 0.0f;
    auto sum_of = [&](const Moments &a) { return a.n > 0.0f ? (double)fmaf(a.n, a.c - c, a.r) : 0.0; };
    double s = sum_of(held);
    for (int e = lane + width; e < count; e += width) s += sum_of(read(e));
    s = all_sum(s, lg);
    const double mean = s * inv;
    const float m = (float)mean;
    float m2 = 0.0f;
    auto add = [&](const Moments &a) {
        // n (sum / n - mean)^2
        const float d = fmaf(a.n, (a.c - c) - m, a.r);
        if (a.n > 0.0f) m2 += fmaf(d * __fdividef(1.0f, a.n), d, a.m2);
    };
    add(held);
    for (int e = lane + width; e < count; e += width) add(read(e));
    return {c, s, mean, all_sum(m2, lg)};
}
// n values with that mean and sum less n c: their mean in fp32, and what is left of their sum.
__device__ __forceinline__ Moments moments_of(float c, double mean, double sum, float m2, float n)
{
    const float own = (float)((double)c + mean);
    return {own, (float)fma(-(double)n, (double)own - (double)c, sum), m2, n};
}
__device__ __forceinline__ void send(const Moments *own, int rank, const Moments &m)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(peer_smem(own, rank)), "f"(m.c), "f"(m.r), "f"(m.m2), "f"(m.n) : "memory");
}

// Shared memory beside the tile: the moments of rows of threads, joined inside the warps where they can be; the groups' moments of every tile of the cluster;
// their means and 1/deviations.
__host__ __device__ __forceinline__ int beside_bytes(const Cut &k)
{
    return (k.rows_of_sums * k.sets + k.groups * (k.tiles < kMaxCluster ? k.tiles : kMaxCluster)) * (int)sizeof(Moments) + k.groups * 8;
}
size_t fwd_beside(const Cut &k) { return (size_t)beside_bytes(k); }
struct Beside {
    Moments *sets, *all;             // [rows][groups * per]; [groups][tiles]
    float *mean, *rstd;
    uint8_t *tile;
    __device__ __forceinline__ Beside(uint8_t *smem, const Cut &k)
    {
        sets = reinterpret_cast<Moments *>(smem);
        all = sets + k.rows_of_sums * k.sets;
        mean = reinterpret_cast<float *>(smem + beside_bytes(k)) - 2 * k.groups;
        rstd = mean + k.groups;
        tile = smem + (beside_bytes(k) + 15) / 16 * 16;
    }
};

// Averages over the sets of u joined channels, in all of them.  (Halves of equal numbers add up to that number.)
template <int V> __device__ __forceinline__ void average_sets(float (&a)[V], int u)
{
#pragma unroll
    for (int w = 1; w < V; w *= 2)
        if (u > w)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if ((i & w) == 0) a[i] = a[i | w] = fmaf(0.5f, a[i], 0.5f * a[i | w]);
}
// What the sums begin with: of a thread's first pixels, up to `head` of `n`, the average.  load(i, f) reads pixel i.
template <int V, typename Load> __device__ __forceinline__ void first_average(float (&f)[V], int head, int n, const Load &load)
{
    load(0, f);
    if (head >= 2 && n >= 4) {
        float g[V];
        load(1, g);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = fmaf(0.5f, f[i], 0.5f * g[i]);
        if (head >= 4) {
            float h[V];
            load(2, g);
            load(3, h);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = fmaf(0.5f, f[i], 0.5f * fmaf(0.5f, g[i], 0.5f * h[i]));
        }
    }
}

// Sums of a thread's pixels: for each set of joined channels those of the differences from an anchor and of their squares.  What their difference q - s^2 / n loses is a
// rounding of q, so q has to be the size of the sum of squares from the mean.  The anchor is the average of the thread's first pixels, of as many as keep n L^2 / head^2 of a first pixel
// that is L from all others to eight times what the group has of it; after every run of kRun pixels it is the mean of all until then.  (With the first value as the anchor
// throughout, 206 pixels lost 2e-4 of the variance, 6900 lost 5e-3.)
template <int V> struct ThreadSums {
    static constexpr int P = V > 1 ? V / 2 : 1;
    two_f32 k[P], s[P], q[P];        // -anchor, sums
    __device__ __forceinline__ void begin(float (&f)[V], int u)
    {
        average_sets(f, u);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            k[i] = two(-f[2 * i < V ? 2 * i : 0], V > 1 ? -f[V > 1 ? 2 * i + 1 : 0] : 0.0f);
            s[i] = q[i] = 0;
        }
    }
    // sums of more pixels, from the same anchor
    __device__ __forceinline__ void begin(const ThreadSums &before)
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            k[i] = before.k[i];
            s[i] = q[i] = 0;
        }
    }
    __device__ __forceinline__ void add(const ThreadSums &more)
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            s[i] = add2(s[i], more.s[i]);
            q[i] = add2(q[i], more.q[i]);
        }
    }
    // the anchor goes to the mean of the n pixels so far
    __device__ __forceinline__ void recentre(int n, int u)
    {
        const float inv = __fdividef(1.0f, (float)n);
        float a[V];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float lo, hi;
            each(mul2(s[i], two(inv, inv)), lo, hi);
            a[2 * i < V ? 2 * i : 0] = lo;
            if (V > 1) a[V > 1 ? 2 * i + 1 : 0] = hi;
        }
        average_sets(a, u);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const two_f32 minus = two(-1.0f, -1.0f), way = two(a[2 * i < V ? 2 * i : 0], V > 1 ? a[V > 1 ? 2 * i + 1 : 0] : 0.0f);
            const two_f32 to = fma2(way, minus, k[i]), moved = fma2(to, minus, k[i]), left = fma2(two(-(float)n, -(float)n), moved, s[i]);
            q[i] = fma2(mul2(moved, minus), add2(s[i], left), q[i]);
            s[i] = left;
            k[i] = to;
        }
    }
    __device__ __forceinline__ void add(const float (&f)[V])
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const two_f32 d = add2(V > 1 ? two(f[2 * i < V ? 2 * i : 0], f[V > 1 ? 2 * i + 1 : 0]) : two(f[0], 0.0f), k[i]);
            s[i] = add2(s[i], d);
            q[i] = fma2(d, d, q[i]);
        }
    }
    // Joined over channels and, where rows of threads lie in a warp, over those: by the first of them to `to`, a thread's sets.  All threads call it.
    __device__ __forceinline__ void store(int n, const Cut &k, bool writes, Moments *to) const
    {
        float ss[V], qq[V], kk[V];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int l = 2 * i < V ? 2 * i : 0, h = V > 1 ? 2 * i + 1 : 0;
            float lo, hi;
            each(s[i], lo, hi); ss[l] = lo; if (V > 1) ss[h] = hi;
            each(q[i], lo, hi); qq[l] = lo; if (V > 1) qq[h] = hi;
            each(this->k[i], lo, hi); kk[l] = lo; if (V > 1) kk[h] = hi;
        }
        if (k.lg_u == 0) store_sets<1>(n, ss, qq, kk, k.least, writes, to);
        if constexpr (V >= 2) if (k.lg_u == 1) store_sets<2>(n, ss, qq, kk, k.least, writes, to);
        if constexpr (V >= 4) if (k.lg_u == 2) store_sets<4>(n, ss, qq, kk, k.least, writes, to);
        if constexpr (V >= 8) if (k.lg_u == 3) store_sets<8>(n, ss, qq, kk, k.least, writes, to);
    }
    template <int U> static __device__ __forceinline__ void store_sets(int n, float (&ss)[V], float (&qq)[V], const float (&kk)[V], int least, bool writes, Moments *to)
    {
        constexpr int Q = V / U;
        // its own: mean, what that leaves of the sum, squares
        float c[Q], r[Q], v[Q];
        const float count = (float)(n * U), inv = n > 0 ? __frcp_rn(count) : 0.0f;
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            float s1 = ss[i * U], q1 = qq[i * U];
#pragma unroll
            for (int j = 1; j < U; ++j) { s1 += ss[i * U + j]; q1 += qq[i * U + j]; }
            const float first = -kk[i * U];
            c[i] = fmaf(s1, inv, first);
            r[i] = fmaf(-count, c[i] - first, s1);
            v[i] = fmaf(-s1 * inv, s1, q1);
            // (an infinity and a NaN stay what they are; a sum of squares is not negative)
            if (v[i] < 0.0f) v[i] = 0.0f;
            if (!(q1 < INFINITY)) v[i] = q1;
        }
        // the warp's, as differences from the mean of the first lane that has these channels
        float all = count;
        if (least < 32) {
            float t[Q], d[Q];
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                const float of = __shfl_sync(0xffffffffu, c[i], (int)threadIdx.x & (least - 1));
                d[i] = n > 0 ? c[i] - of : 0.0f;
                t[i] = n > 0 ? fmaf(count, d[i], r[i]) : 0.0f;
                c[i] = of;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                if (o >= least) {
                    all += __shfl_xor_sync(0xffffffffu, all, o);
#pragma unroll
                    for (int i = 0; i < Q; ++i) t[i] += __shfl_xor_sync(0xffffffffu, t[i], o);
                }
            const float inv_all = all > 0.0f ? __fdividef(1.0f, all) : 0.0f;
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                const float mean = t[i] * inv_all, e = fmaf(count, d[i] - mean, r[i]);
                if (n > 0) v[i] = fmaf(e * inv, e, v[i]);
                const float of = c[i];
                c[i] = of + mean;
                r[i] = fmaf(-all, c[i] - of, t[i]);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                if (o >= least)
#pragma unroll
                    for (int i = 0; i < Q; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        }
        if (writes)
#pragma unroll
            for (int i = 0; i < Q; ++i) to[i] = {c[i], r[i], v[i], all};
    }
};

// The block's groups from its sets; write(g, lane, width, moments) is called by the lanes of a group, that many, with the same moments.  Called by all.
template <int V, typename Write> __device__ __forceinline__ void join_groups(const Tile<V> &t, const Cut &k, const Moments *sets, Write write)
{
    const int sets_of = k.pieces > 1 ? t.cs >> k.lg_u : k.per, count = sets_of * k.rows_of_sums, across = k.sets;
    const float n = (float)t.rows * (float)(k.pieces > 1 ? t.cs : k.Cg);
    const float inv = n > 0.0f ? __fdividef(1.0f, n) : 0.0f;
    const int lg = k.lg_tile, width = 1 << lg, mine = threadIdx.x >> lg, lane = threadIdx.x & (width - 1);
    // (a warp without a group has nothing to do)
    for (int g0 = 0; g0 + (int)((threadIdx.x & ~31u) >> lg) < k.groups; g0 += kGnThreads >> lg) {
        const int g = g0 + mine;
        const Joined a = join(lane, lg, g < k.groups ? count : 0, (double)inv, [&](int e) {
            const int y = k.pieces > 1 ? e / sets_of : (int)k.by_per((uint32_t)e);
            return sets[y * across + g * k.per + e - y * sets_of];
        });
        if (g < k.groups) write(g, lane, width, moments_of(a.c, a.mean, a.sum, a.m2, n));
    }
}

// Pixels that are worked on at once: SiLU's reciprocals serve two.
template <int ACT> constexpr int kAtOnce = ACT == kSilu ? 2 : 1;
// Of two channels of J pixels.
template <int ACT, int J> __device__ __forceinline__ void activate(two_f32 (&z)[J])
{
    if (ACT != kNone)
#pragma unroll
        for (int j = 0; j < J; ++j) z[j] = at_least2(z[j], ACT == kRelu ? 0.0f : kLeastZ);
    if (ACT == kSilu) {
        two_f32 e[J], f[J];
        sigmoids(z, e, f);
#pragma unroll
        for (int j = 0; j < J; ++j) z[j] = mul2(z[j], f[j]);
    }
}
// Of one channel of two pixels.
__device__ __forceinline__ two_f32 silu(two_f32 z)
{
    float t0, t1, s0, s1;
    z = at_least2(z, kLeastZ);
    each(mul2(z, two(kMinusLog2e, kMinusLog2e)), t0, t1);
    each(fma2(two(ex2(t0), ex2(t1)), two(1.0f, 0x1p-126f), two(1.0f, 0x1p-126f)), s0, s1);
    const float r = reciprocal(s0 * s1);
    return mul2(z, two(r * s1, r * s0 * 0x1p-126f));
}

// (gamma and beta may lie on any multiple of four bytes)
template <int V> __device__ __forceinline__ void load_channels(float (&f)[V], const float *p, const Tile<V> &t, float none)
{
    if (p && t.has()) {
        load_floats(f, p + t.channel());
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = none;
    }
}

// What the outputs of a thread's channels are made with.
template <int V> struct Affine {
    static constexpr int P = V > 1 ? V / 2 : 1;
    two_f32 m[P], a[P], b[P];        // -mean, rstd gamma, beta
    __device__ __forceinline__ Affine(const GnFwd &p, const Tile<V> &t, const float (&ga)[V], const float (&be)[V], const float *mean, const float *rstd)
    {
        float mm[V], aa[V];
        const bool one = p.cut.Cg % V == 0;          // group
        int g = p.cut.pieces > 1 ? 0 : (int)p.cut.by_group((uint32_t)(t.tx * V));
        float m0 = -mean[g], r0 = rstd[g];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (i > 0 && !one) {
                g = (int)p.cut.by_group((uint32_t)(t.tx * V + i));
                m0 = -mean[g];
                r0 = rstd[g];
            }
            mm[i] = m0;
            aa[i] = r0 * ga[i];
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int j = V > 1 ? 2 * i + 1 : 0;
            m[i] = two(mm[2 * i < V ? 2 * i : 0], mm[j]);
            a[i] = two(aa[2 * i < V ? 2 * i : 0], aa[j]);
            b[i] = two(be[2 * i < V ? 2 * i : 0], be[j]);
        }
    }
    // Of J pixels.
    template <int ACT, int J, typename TX> __device__ __forceinline__ void operator()(const Vec<TX, V> (&v)[J], float (&y)[J][V]) const
    {
        float x[J][V];
#pragma unroll
        for (int j = 0; j < J; ++j) v[j].get(x[j]);
        if constexpr (V == 1 && J == 2) {
            // (one channel: the two pixels are a pair)
            each(silu(fma2(add2(two(x[0][0], x[1][0]), m[0]), a[0], b[0])), y[0][0], y[1][0]);
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int l = 2 * i < V ? 2 * i : 0, h = V > 1 ? 2 * i + 1 : 0;
                two_f32 z[J];
#pragma unroll
                for (int j = 0; j < J; ++j) z[j] = fma2(add2(two(x[j][l], x[j][h]), m[i]), a[i], b[i]);
                activate<ACT, J>(z);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    float y0, y1;
                    each(z[j], y0, y1);
                    y[j][l] = y0;
                    if (V > 1) y[j][h] = y1;
                }
            }
        }
    }
};

// Mean and 1/deviation of the block's groups, the first of them group `first` of all images', from their parts, which read(g, e) gives for e < count.  All threads call it.
template <typename Read> __device__ __forceinline__ void finish_groups(const GnFwd &P, int groups, int count, bool write, long long first, float *mean, float *rstd, Read read)
{
    const int lg = P.cut.lg_slab, mine = threadIdx.x >> lg, lane = threadIdx.x & ((1 << lg) - 1);
    for (int g0 = 0; g0 + (int)((threadIdx.x & ~31u) >> lg) < groups; g0 += kGnThreads >> lg) {
        const int g = g0 + mine;
        const Joined a = join(lane, lg, g < groups ? count : 0, P.cut.inv_n, [&](int e) { return read(g, e); });
        if (g < groups && lane == 0) {
            mean[g] = (float)((double)a.c + a.mean);
            rstd[g] = __frsqrt_rn(fmaf(a.m2, (float)P.cut.inv_n, P.eps));
            if (write) {
                if (P.mean) P.mean[first + g] = mean[g];
                if (P.rstd) P.rstd[first + g] = rstd[g];
            }
        }
    }
    __syncthreads();
}

template <typename TX, typename TY, int V, int ACT>
__device__ __forceinline__ void apply_tile(const GnFwd &P, const Tile<V> &t, const Affine<V> &affine, const TX *slots)
{
    TY *y = static_cast<TY *>(P.Y) + (t.b * P.cut.HW + t.first + t.ty) * P.ldy + t.channel();
    const long long step = t.R * P.ldy;
    constexpr int J = kAtOnce<ACT>;
    auto work = [&](int i, auto pixels) {
        constexpr int n = decltype(pixels)::value;
        Vec<TX, V> v[n];
        float o[n][V];
#pragma unroll
        for (int j = 0; j < n; ++j) v[j].load(slots + (i + j) * (kGnThreads * V));
        affine.template operator()<ACT, n>(v, o);
#pragma unroll
        for (int j = 0; j < n; ++j) store(y + (i + j) * step, o[j]);
    };
    int i = 0;
#pragma unroll (4 / J)
    for (; i + J <= t.n; i += J) work(i, std::integral_constant<int, J>());
    if (J > 1 && i < t.n) work(i, std::integral_constant<int, 1>());
}

// 64 x 12544 x 64 bf16 with a ReLU in 50 us, 4.1 TB/s: bound by latency.  Two blocks of 8 warps an SM issue on 39 % of the cycles, and half of what they issue joins sums; a
// seventh of the SMs' room for warps is empty, as clusters of eight leave some and 128 of them are 3.5 rounds.
// ---- resident -----------------------------------------------------------------------------------------------------------------
template <typename TX, typename TY, int V>
__global__ void __launch_bounds__(kGnThreads, 2) gn_fwd_kernel(const __grid_constant__ GnFwd P)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const Tile<V> t(P.cut, blockIdx.x);
    const Beside at(smem, P.cut);
    const int u = 1 << P.cut.lg_u, tiles = P.cut.tiles, groups = P.cut.groups;
    pdl_begin();
    if (tiles > 1) arrive_first();
    TX *const slots = reinterpret_cast<TX *>(at.tile) + threadIdx.x * V;
    {
        const TX *from = static_cast<const TX *>(P.X) + (t.b * P.cut.HW + t.first + t.ty) * P.ldx + t.channel();
        const long long step = t.R * P.ldx;
        int begin = 0;
#pragma unroll
        for (int q = 0; q < kShares; ++q) {
            const int end = share_end(t.n, q);
            copy_vectors<TX, V>(slots + begin * (kGnThreads * V), from + begin * step, step, end - begin);
            end_share();
            begin = end;
        }
    }
    float ga[V], be[V];
    load_channels(ga, P.gamma, t, 1.0f);
    load_channels(be, P.beta, t, 0.0f);
    {
        constexpr bool kRuns = kTileMost / (kGnThreads * V * sizeof(TX)) > kRun;      // of more than one
        ThreadSums<V> sums, run;
        int next = kRun;
        auto load = [&](int i, float (&f)[V]) {
            Vec<TX, V> v;
            v.load(slots + i * (kGnThreads * V));
            v.get(f);
        };
        as_they_come(t.n, 0, [&](int begin, int end) {
            if (begin == 0) {
                float f[V] = {};
                if (end > 0) first_average(f, P.cut.head, end, load);
                sums.begin(f, u);
                if (kRuns) run.begin(sums);
            }
            for (int i = begin; i < end;) {
                const int stop = kRuns ? min(end, next) : end;
#pragma unroll 4
                for (; i < stop; ++i) {
                    float f[V];
                    load(i, f);
                    if (kRuns) run.add(f);
                    else sums.add(f);
                }
                if (kRuns && i == next) {
                    sums.add(run);
                    sums.recentre(i, u);
                    run.begin(sums);
                    next += kRun;
                }
            }
        });
        if (kRuns) sums.add(run);
        const int y = P.cut.joint > 1 ? (int)(threadIdx.x >> 5) : t.ty;
        sums.store(t.n, P.cut, P.cut.joint > 1 ? (int)(threadIdx.x & 31) < P.cut.least : t.has(), at.sets + y * P.cut.sets + t.tx * (V >> P.cut.lg_u));
    }
    __syncthreads();
    if (tiles > 1) wait_for_all();                   // all blocks are there
    // to all blocks of the cluster
    join_groups(t, P.cut, at.sets, [&](int g, int lane, int width, const Moments &of) {
        if (tiles == 1) {
            if (lane == 0) at.all[g] = of;
        } else {
            for (int to = lane; to < tiles; to += width) send(at.all + g * tiles + t.tile, to, of);
        }
    });
    if (tiles == 1) {
        __syncthreads();
    } else {
        arrive();
        wait_for_all();
    }
    finish_groups(P, groups, tiles, t.tile == 0, t.b * P.cut.G + (int)P.cut.by_group((uint32_t)t.c0), at.mean, at.rstd, [&](int g, int k) { return at.all[g * tiles + k]; });
    if (t.n > 0) {
        const Affine<V> affine(P, t, ga, be, at.mean, at.rstd);
        if (P.act == kSilu) apply_tile<TX, TY, V, kSilu>(P, t, affine, slots);
        else if (P.act == kRelu) apply_tile<TX, TY, V, kRelu>(P, t, affine, slots);
        else apply_tile<TX, TY, V, kNone>(P, t, affine, slots);
    }
}

// 131072 pixels of 512 channels, one group of 67 million values, in 121 us: three passes over 134 MB would take 61.
// ---- two reads ----------------------------------------------------------------------------------------------------------------
template <typename TX, int V>
__global__ void __launch_bounds__(kGnThreads) gn_sums_kernel(const __grid_constant__ GnFwd P)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const Tile<V> t(P.cut, blockIdx.x);
    Moments *const sets = reinterpret_cast<Moments *>(smem);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int u = 1 << P.cut.lg_u;
    {
        const TX *x = static_cast<const TX *>(P.X) + (t.b * P.cut.HW + t.first + t.ty) * P.ldx + t.channel();
        const long long step = t.R * P.ldx;
        ThreadSums<V> sums = {};
        Vec<TX, V> v;
        float f[V];
        auto load = [&](int i, float (&f)[V]) {
            v.load(x + i * step);
            v.get(f);
        };
        if (t.n < 8) {
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = 0.0f;
            if (t.n > 0) first_average(f, P.cut.head, t.n, load);
            sums.begin(f, u);
        }
        for (int i = 0; i < t.n;) {
            const int end = min(t.n, i + kRun);
            ThreadSums<V> run;
            run.begin(sums);
            for (; i + 8 <= end; i += 8) {
                Vec<TX, V> w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j].load(x + (i + j) * step);
                if (i == 0) {
                    // (of those that are there already: with loads of their own 16 x 65536 x 24 fp32 took 72.4 us for 70.3)
                    first_average(f, P.cut.head, 8, [&](int j, float (&g)[V]) { w[j].get(g); });
                    sums.begin(f, u);
                    run.begin(sums);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    w[j].get(f);
                    run.add(f);
                }
            }
            for (; i < end; ++i) {
                load(i, f);
                run.add(f);
            }
            sums.add(run);
            if (end < t.n) sums.recentre(end, u);
        }
        const int y = P.cut.joint > 1 ? (int)(threadIdx.x >> 5) : t.ty;
        sums.store(t.n, P.cut, P.cut.joint > 1 ? (int)(threadIdx.x & 31) < P.cut.least : t.has(), sets + y * P.cut.sets + t.tx * (V >> P.cut.lg_u));
    }
    __syncthreads();
    // one part of each group for the tile
    const int g0 = t.c0 / P.cut.Cg, piece = P.cut.pieces > 1 ? (t.c0 - g0 * P.cut.Cg) / P.cut.slab : 0;
    join_groups(t, P.cut, sets, [&](int g, int lane, int, const Moments &m) {
        if (lane == 0) P.parts[((t.b * P.cut.G + g0 + g) * P.cut.pieces + piece) * P.cut.tiles + t.tile] = m;
    });
}

template <typename TX, typename TY, int V, int ACT>
__device__ __forceinline__ void apply_rows(const GnFwd &P, const Tile<V> &t, const Affine<V> &affine)
{
    const TX *x = static_cast<const TX *>(P.X) + (t.b * P.cut.HW + t.first + t.ty) * P.ldx + t.channel();
    TY *y = static_cast<TY *>(P.Y) + (t.b * P.cut.HW + t.first + t.ty) * P.ldy + t.channel();
    const long long in = t.R * P.ldx, out = t.R * P.ldy;
    constexpr int J = kAtOnce<ACT>;
    int i = 0;
    for (; i + 8 <= t.n; i += 8) {
        Vec<TX, V> w[8 / J][J];
        float o[J][V];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j / J][j % J].load(x + (i + j) * in);
#pragma unroll
        for (int j = 0; j < 8; j += J) {
            affine.template operator()<ACT, J>(w[j / J], o);
#pragma unroll
            for (int k = 0; k < J; ++k) store(y + (i + j + k) * out, o[k]);
        }
    }
    for (; i < t.n; ++i) {
        Vec<TX, V> v[1];
        float o[1][V];
        v[0].load(x + i * in);
        affine.template operator()<ACT, 1>(v, o);
        store(y + i * out, o[0]);
    }
}
template <typename TX, typename TY, int V>
__global__ void __launch_bounds__(kGnThreads) gn_apply_kernel(const __grid_constant__ GnFwd P)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const Tile<V> t(P.cut, blockIdx.x);
    float ga[V], be[V];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    load_channels(ga, P.gamma, t, 1.0f);
    load_channels(be, P.beta, t, 0.0f);
    const int groups = P.cut.groups, count = P.cut.pieces * P.cut.tiles;
    float *const mean = reinterpret_cast<float *>(smem), *const rstd = mean + groups;
    const long long first = t.b * P.cut.G + t.c0 / P.cut.Cg;
    finish_groups(P, groups, count, t.tile == 0 && t.c0 % P.cut.Cg == 0, first, mean, rstd, [&](int g, int k) { return P.parts[(first + g) * count + k]; });
    if (t.n == 0) return;
    const Affine<V> affine(P, t, ga, be, mean, rstd);
    if (P.act == kSilu) apply_rows<TX, TY, V, kSilu>(P, t, affine);
    else if (P.act == kRelu) apply_rows<TX, TY, V, kRelu>(P, t, affine);
    else apply_rows<TX, TY, V, kNone>(P, t, affine);
}

// ---- host -----------------------------------------------------------------------------------------------------------------------
size_t parts_bytes(const Cut &k, long long tiles) { return (size_t)tiles * k.G * k.pieces * sizeof(Moments); }

template <typename TX, typename TY, int V> int fwd(GnFwd &P, const Plan &plan, long long B, const twn_device_info &dev, void *workspace, cudaStream_t s)
{
    const Cut &k = P.cut;
    if (plan.resident) {
        static bool done[64] = {false};
        const int rc = allow_tile(gn_fwd_kernel<TX, TY, V>, dev.ordinal, done);
        if (rc != TWN_OK) return rc;
        TWN_CUDA_OK(launch_clusters(gn_fwd_kernel<TX, TY, V>, B * k.slabs * k.tiles, k.tiles, plan.smem, s, P));
        return TWN_OK;
    }
    P.parts = static_cast<Moments *>(workspace);
    const int grid = (int)(B * k.slabs * k.tiles);
    TWN_CUDA_OK(twn_launch_pdl(true, gn_sums_kernel<TX, V>, grid, kGnThreads, (size_t)k.rows_of_sums * k.sets * sizeof(Moments), s, P));
    TWN_CUDA_OK(twn_launch_pdl(true, gn_apply_kernel<TX, TY, V>, grid, kGnThreads, (size_t)k.groups * 8, s, P));
    return TWN_OK;
}
template <typename TX, typename TY> int fwd_any(GnFwd &P, const Plan &plan, long long B, int V, const twn_device_info &dev, void *workspace, cudaStream_t s)
{
    if constexpr (sizeof(TX) + sizeof(TY) == 4)
        if (V == 8) return fwd<TX, TY, 8>(P, plan, B, dev, workspace, s);
    if (V == 4) return fwd<TX, TY, 4>(P, plan, B, dev, workspace, s);
    if (V == 2) return fwd<TX, TY, 2>(P, plan, B, dev, workspace, s);
    return fwd<TX, TY, 1>(P, plan, B, dev, workspace, s);
}

}  // namespace

extern "C" size_t twn_group_norm_fwd_workspace_bytes(int64_t B, int64_t HW, int64_t C, int32_t groups)
{
    if (check_groups(B, HW, C, groups) != TWN_OK || B == 0 || HW == 0) return 0;
    size_t most = 0;
    for (int V : {1, 2, 4, 8}) {
        Cut k = cut_of(HW, (int)C, groups);
        if (C % V || !vectors_fit(k.Cg, V) || !cut_streamed(k, B, V)) continue;
        most = std::max(most, parts_bytes(k, tiles_at_most(k, B, V, false)));
    }
    return (most + 255) / 256 * 256;
}

extern "C" int twn_group_norm_fwd(const void *X, int32_t x_dtype, int64_t ldx, int64_t B, int64_t HW, int64_t C, int32_t groups, const float *gamma,
                                  const float *beta, double eps, int32_t act, void *Y, int32_t y_dtype, int64_t ldy, float *mean, float *rstd,
                                  void *workspace, size_t workspace_bytes, twn_stream_t stream)
{
    int rc = check_groups(B, HW, C, groups);
    if (rc != TWN_OK) return rc;
    TWN_REQUIRE(is_act(act) && std::isfinite(eps) && eps >= 0.0, TWN_ERR_INVALID_ARG);
    const long long M = B * HW;
    rc = check_matrix(X, x_dtype, ldx, M, C);
    if (rc == TWN_OK) rc = check_matrix(Y, y_dtype, ldy, M, C);
    if (rc != TWN_OK) return rc;
    for (const void *p : {(const void *)gamma, (const void *)beta, (const void *)mean, (const void *)rstd}) TWN_REQUIRE(twn_aligned(p, 4), TWN_ERR_MISALIGNED);
    if (M == 0) return TWN_OK;
    Cut k = cut_of(HW, (int)C, groups);
    const int V = widest(x_dtype == TWN_BF16 && y_dtype == TWN_BF16 ? 8 : 4, (int)C, k.Cg,
                         [&](int v) { return vector_rows(X, x_dtype, ldx, v) && vector_rows(Y, y_dtype, ldy, v); });
    Plan p;
    rc = plan(k, p, B, V, (int)size_of(x_dtype), (int)size_of(x_dtype), fwd_beside);
    if (rc != TWN_OK) return rc;
    // (a tile in shared memory needs none of it)
    const size_t need = std::max<size_t>(256, p.resident ? 0 : parts_bytes(k, B * k.tiles));
    TWN_REQUIRE(workspace != nullptr && workspace_bytes >= need, TWN_ERR_WORKSPACE);
    TWN_REQUIRE(twn_aligned(workspace, 256), TWN_ERR_MISALIGNED);
    Places places;
    places.matrix(Y, y_dtype, ldy, M, C, true);
    places.matrix(X, x_dtype, ldx, M, C, false);
    for (const void *q : {(const void *)gamma, (const void *)beta}) places.vector(q, 4 * C, false);
    for (const void *q : {(const void *)mean, (const void *)rstd}) places.vector(q, 4 * B * groups, true);
    places.vector(workspace, (long long)need, true);
    TWN_REQUIRE(places.apart(), TWN_ERR_INVALID_ARG);
    twn_device_info dev;
    rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    GnFwd P = {X, Y, gamma, beta, mean, rstd, nullptr, ldx, ldy, k, act, (float)eps};
    cudaStream_t s = twn_cu(stream);
#define TWN_GN_FWD(TX, TY) fwd_any<TX, TY>(P, p, B, V, dev, workspace, s)
    if (x_dtype == TWN_BF16) return y_dtype == TWN_BF16 ? TWN_GN_FWD(bf16, bf16) : TWN_GN_FWD(bf16, float);
    return y_dtype == TWN_BF16 ? TWN_GN_FWD(float, bf16) : TWN_GN_FWD(float, float);
#undef TWN_GN_FWD
}
