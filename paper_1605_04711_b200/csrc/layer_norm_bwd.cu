// Layer norm, backward (see layer_norm.cuh).
#include "layer_norm.cuh"

namespace {

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
// warps of a block took 10 of 29 us for rows of 64).
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

// Rows of more than 8192 elements, through shared memory by bulk copies (see norm_fwd_ring_kernel; up to 8192 it is behind the one above by up to 1.6 times).
// A block is one team of at least 288 threads, and has a row at a time.  The sums over the rows fill the registers, so a row is read twice
// from its stage, for its two sums and for its gradient; the stage is refilled after the next row's sums, when the whole team has left it.
template <typename TD, typename TX, typename TO, int V, int E, int TT>
__global__ void __launch_bounds__(kBwdThreads, 1) norm_bwd_ring_kernel(const __grid_constant__ BwdParams P, const __grid_constant__ Ring R)
{
    constexpr int P2 = E / 2, W = V;         // elements worked on at a time
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ unsigned long long full[kMaxRing];
    __shared__ __align__(16) float red[2][32][2];
    __shared__ volatile int gave_up;
    unsigned int turn = 0;
    const int T = TT ? TT : P.T, t = threadIdx.x, C = TT ? TT * E : (int)P.C;
    const float inv = 1.0f / (float)C;
    const Columns<V, TT> col{T, t, C};
    if (t == 0) {
        for (int s = 0; s < R.stages; ++s) mbar_init(&full[s], 1);
        gave_up = 0;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    pdl_begin();
    uint8_t *const stages = ring + R.params;
    const long long first = blockIdx.x, step = gridDim.x;
    auto issue = [&](long long r, int s) {
        if (r >= P.M) return;
        uint8_t *const st = stages + (size_t)s * R.stage_bytes;
        mbar_expect_tx(&full[s], C * (uint32_t)(sizeof(TD) + sizeof(TX)));
        bulk_load(st, static_cast<const TD *>(P.dY) + r * P.lddy, C * (uint32_t)sizeof(TD), &full[s]);
        bulk_load(st + R.second, static_cast<const TX *>(P.X) + r * P.ldx, C * (uint32_t)sizeof(TX), &full[s]);
    };
    if (t == 0)
        for (int s = 0; s < R.stages; ++s) issue(first + s * step, s);
    const bool in_ring = TT ? TT * E * sizeof(float) <= kBwdRingBytes / 2 : R.params > 0;
    float *const gammas = in_ring ? reinterpret_cast<float *>(ring) : nullptr;
    if (in_ring) {
        for (int c = threadIdx.x; c < C; c += T) gammas[param_at<V>(c, C)] = P.gamma ? P.gamma[c] : 1.0f;
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
        const bool ok = row_is_there(&full[s], ph, &gave_up);
        const uint8_t *const st = stages + (size_t)s * R.stage_bytes;
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
        if (!ok) drop_sums(a_g, a_b);
        float sums[2] = {sum2(s0), ok ? sum2(s1) : __uint_as_float(0x7FC00000u)};
        if constexpr (TT > 0) team_sum<TT>(sums, red, turn, 0);
        else team_sum(sums, T, red, turn, 0);
        // the whole team has left the row before this one: its stage is free
        if (t == 0 && r != first && ok) issue(r + (R.stages - 1) * step, s == 0 ? R.stages - 1 : s - 1);
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
    leave_rows(&gave_up);
    if (P.part == nullptr) return;
    float g[E], b[E];
#pragma unroll
    for (int i = 0; i < P2; ++i) { each(a_g[i], g[2 * i], g[2 * i + 1]); each(a_b[i], b[2 * i], b[2 * i + 1]); }
    join_sums<V>(g, b, col, true, 0, 1, nullptr, P.part + (long long)blockIdx.x * 2 * C);
}

// Long rows, first pass: sum(g) / C and sum(g xh) / C of every row, a thread's vectors added in fp64 (see norm_fwd_long_kernel).
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
        double total[2] = {0.0, 0.0};
        for (long long col = (long long)threadIdx.x * V; col < P.C; col += kBwdThreads * V) {
            Vec<TD, V> vd;
            Vec<TX, V> vx;
            float d[V], x[V], ga[V], v_sum[2] = {0.0f, 0.0f};
            vd.load(dy + col);
            vx.load(xr + col);
            vd.get(d);
            vx.get(x);
            load_param(ga, P.gamma, col, 1.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float g = d[i] * ga[i];
                v_sum[0] += g;
                v_sum[1] = fmaf(g, (x[i] - mean) * rstd, v_sum[1]);
            }
            total[0] += (double)v_sum[0];
            total[1] += (double)v_sum[1];
        }
        float s[2] = {(float)total[0], (float)total[1]};
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
// W columns a thread, so that up to 4736 channels, or 9472, are a block an SM, which may start early: while the launch before it still writes the parts,
// so their loads are plain ones, not those of data that nobody writes.
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
                const float4 a = *reinterpret_cast<const float4 *>(from);
                w[k][0] = a.x; w[k][1] = a.y; w[k][2] = a.z; w[k][3] = a.w;
            } else if constexpr (W == 2) {
                const float2 a = *reinterpret_cast<const float2 *>(from);
                w[k][0] = a.x; w[k][1] = a.y;
            } else {
                w[k][0] = *from;
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

template <typename TD, typename TX, typename TO, int V, int E, int TT>
int launch_bwd_ring(const BwdParams &P, const RingShape &r, const twn_device_info &dev, cudaStream_t s)
{
    static bool done[64] = {false};
    const int rc = allow_ring(norm_bwd_ring_kernel<TD, TX, TO, V, E, TT>, dev.ordinal, done);
    if (rc != TWN_OK) return rc;
    TWN_CUDA_OK(twn_launch_small(norm_bwd_ring_kernel<TD, TX, TO, V, E, TT>, P.parts, r.T, r.smem, s, P, r.ring));
    return TWN_OK;
}
template <typename TD, typename TX, typename TO, int V, int E> bool bwd_ring(BwdParams &P, const twn_device_info &dev, cudaStream_t s, int &rc)
{
    RingShape r;
    const size_t second = P.C * sizeof(TD);
    if (!ring_shape(r, kBwdRingBytes, P.C, E, kBwdThreads, second + P.C * sizeof(TX), second, sizeof(float) * P.C)) return false;
    P.T = r.T;
    P.parts = (int)std::min<long long>(P.M, std::min(dev.sm_count, kPartBlocks));
    const int filled = P.C == (long long)r.T * E ? r.T : 0;
    rc = filled == 512 ? launch_bwd_ring<TD, TX, TO, V, E, 512>(P, r, dev, s) : launch_bwd_ring<TD, TX, TO, V, E, 0>(P, r, dev, s);
    return true;
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
    Places places;
    if (M > 0) {
        places.matrix(dX, dx_dtype, lddx, M, C, true);
        places.matrix(dY, dy_dtype, lddy, M, C, false);
        places.matrix(X, x_dtype, ldx, M, C, false);
        places.matrix(residual, dx_dtype, lddx, M, C, false);
        for (const void *p : {(const void *)mean, (const void *)rstd}) places.vector(p, 4 * M, false);
    }
    places.vector(gamma, 4 * C, false);
    for (const void *p : {(const void *)dgamma, (const void *)dbeta}) places.vector(p, 4 * C, true);
    places.vector(workspace, (long long)twn_layer_norm_bwd_workspace_bytes(M, C), true);
    TWN_REQUIRE(places.apart(), TWN_ERR_INVALID_ARG);
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
