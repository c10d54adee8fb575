// Layer norm, forward (see layer_norm.cuh).
#include "layer_norm.cuh"

namespace {

struct FwdParams {
    const void *X;
    void *Y;
    const float *gamma, *beta;
    float *mean, *rstd;
    long long ldx, ldy, M, C;
    float eps;
    int T;
};

constexpr int kFwdThreads = 512;             // of a block, but for teams of 1024

// One row per team, in registers.  C <= T * E.  MANY: teams of more than a warp share a block, with a named barrier each; the number of a barrier that is not
// known at compile time takes all sixteen, and fewer small blocks fit an SM (10000 rows of 1001: 46 us for 22.7 of a block a team).
template <typename TX, typename TY, int V, int E, int TT, bool MANY>
__global__ void __launch_bounds__(MANY || TT <= 32 ? kFwdThreads : TT, TT <= 32 || V == 1 ? 1 : MANY ? 2 : 1024 / (TT ? TT : 1)) norm_fwd_kernel(const __grid_constant__ FwdParams P)
{
    constexpr int NV = E / V, P2 = E / 2;
    __shared__ __align__(16) float red[2][32][2];
    unsigned int turn = 0;
    const int T = TT ? TT : P.T, t = threadIdx.x & (T - 1), C = (int)P.C;
    const int teams = blockDim.x / T, team = threadIdx.x / T, barrier = MANY ? team + 1 : 0;
    const float inv = 1.0f / (float)C;
    const Columns<V, TT> col{T, t, C};
    pdl_begin();
    for (long long r0 = (long long)blockIdx.x * teams; r0 < P.M; r0 += (long long)gridDim.x * teams) {
        const long long r = r0 + team;
        const bool live = r < P.M;
        const TX *x = static_cast<const TX *>(P.X) + (live ? r : 0) * P.ldx;
        Vec<TX, V> raw[NV];
        load_vectors(raw, x, col, live);
        two_f32 d[P2], s2 = 0, q2 = 0;
        {
            float f[E];
#pragma unroll
            for (int j = 0; j < NV; ++j) raw[j].get(*reinterpret_cast<float(*)[V]>(f + j * V));
#pragma unroll
            for (int i = 0; i < P2; ++i) {
                d[i] = two(f[2 * i], f[2 * i + 1]);
                s2 = add2(s2, d[i]);
            }
        }
        float s[1] = {sum2(s2)};
        if constexpr (TT > 0) team_sum<TT>(s, red, turn, barrier);
        else team_sum(s, T, red, turn, barrier);
        const float mean = s[0] * inv;
        const two_f32 minus = two(-mean, -mean);
#pragma unroll
        for (int i = 0; i < P2; ++i) d[i] = add2(d[i], minus);
        // nothing of what is past the row's end
        constexpr int K = NV < 8 ? NV : 8;
#pragma unroll
        for (int j0 = 0; j0 < NV; j0 += K)
            if (!col.whole(j0 + K - 1))
#pragma unroll
                for (int i = j0 * V / 2; i < (j0 + K) * V / 2; ++i) {
                    if (V > 1) {
                        if (col(2 * i / V) >= C) d[i] = 0;
                    } else {
                        float a, b;
                        each(d[i], a, b);
                        d[i] = two(col(2 * i) < C ? a : 0.0f, col(2 * i + 1) < C ? b : 0.0f);
                    }
                }
#pragma unroll
        for (int i = 0; i < P2; ++i) q2 = fma2(d[i], d[i], q2);
        float q[1] = {sum2(q2)};
        if constexpr (TT > 0) team_sum<TT>(q, red, turn, barrier);
        else team_sum(q, T, red, turn, barrier);
        const float rstd = rsqrtf(fmaf(q[0], inv, P.eps));
        if (!live) continue;
        const two_f32 scale = two(rstd, rstd);
        TY *y = static_cast<TY *>(P.Y) + r * P.ldy;
        // K vectors: whole where the team's are, so that their loads of gamma and beta go together
        auto put = [&](int j, const float(&ga)[V], const float(&be)[V]) {
            float o[V];
            if constexpr (V > 1) {
#pragma unroll
                for (int i = 0; i < V / 2; ++i)
                    each(fma2(mul2(d[j * V / 2 + i], scale), two(ga[2 * i], ga[2 * i + 1]), two(be[2 * i], be[2 * i + 1])), o[2 * i], o[2 * i + 1]);
            } else {
                float a, b;
                each(d[j / 2], a, b);
                o[0] = fmaf((j & 1 ? b : a) * rstd, ga[0], be[0]);
            }
            store(y + col(j), o);
        };
#pragma unroll
        for (int j0 = 0; j0 < NV; j0 += K) {
            const bool whole = col.whole(j0 + K - 1);
            if (whole && V == 1) {
                float ga[K][V], be[K][V];
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    load_param(ga[j], P.gamma, col(j0 + j), 1.0f);
                    load_param(be[j], P.beta, col(j0 + j), 0.0f);
                }
#pragma unroll
                for (int j = 0; j < K; ++j) put(j0 + j, ga[j], be[j]);
            } else {
#pragma unroll
                for (int j = j0; j < j0 + K; ++j) {
                    if (!whole && col(j) >= C) continue;
                    float ga[V], be[V];
                    load_param(ga, P.gamma, col(j), 1.0f);
                    load_param(be, P.beta, col(j), 0.0f);
                    put(j, ga, be);
                }
            }
        }
        if (t == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
    }
}

template <int E> constexpr int fwd_ring_threads() { return E >= 64 ? 512 : E >= 32 ? 768 : 1024; }

// TT > 0: teams of TT threads whose elements the row fills, C = TT E, so that addresses are constants and nothing is checked.
template <typename TX, typename TY, int V, int E, int TT>
__global__ void __launch_bounds__(fwd_ring_threads<E>(), 1) norm_fwd_ring_kernel(const __grid_constant__ FwdParams P, const __grid_constant__ Ring R)
{
    constexpr int NV = E / V, P2 = E / 2;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ unsigned long long full[kMaxTeams][kMaxRing];
    __shared__ __align__(16) float red[2][32][2];
    __shared__ volatile int gave_up;
    unsigned int turn = 0;
    const int T = TT ? TT : P.T, team = threadIdx.x / T, t = threadIdx.x - team * T, C = TT ? TT * E : (int)P.C;
    const int teams = blockDim.x / T, barrier = teams > 1 ? team + 1 : 0;
    const float inv = 1.0f / (float)C;
    const Columns<V, TT> col{T, t, C};
    if (t == 0)
        for (int s = 0; s < R.stages; ++s) mbar_init(&full[team][s], 1);
    if (threadIdx.x == 0) gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    pdl_begin();
    uint8_t *const mine = ring + R.params + (size_t)team * R.stages * R.stage_bytes;
    const long long first = (long long)blockIdx.x * teams + team, step = (long long)gridDim.x * teams;
    auto issue = [&](long long r, int s) {
        if (r >= P.M) return;
        mbar_expect_tx(&full[team][s], C * (uint32_t)sizeof(TX));
        bulk_load(mine + (size_t)s * R.stage_bytes, static_cast<const TX *>(P.X) + r * P.ldx, C * (uint32_t)sizeof(TX), &full[team][s]);
    };
    if (t == 0)
        for (int s = 0; s < R.stages; ++s) issue(first + s * step, s);
    const bool in_ring = TT ? 2 * TT * E * sizeof(float) <= kFwdRingBytes / 2 : R.params > 0;
    float *const gammas = in_ring ? reinterpret_cast<float *>(ring) : nullptr, *const betas = in_ring ? gammas + C : nullptr;
    if (in_ring) {
        for (int c = threadIdx.x; c < C; c += blockDim.x) {
            gammas[param_at<V>(c, C)] = P.gamma ? P.gamma[c] : 1.0f;
            betas[param_at<V>(c, C)] = P.beta ? P.beta[c] : 0.0f;
        }
        __syncthreads();
    }
    int s = 0;
    uint32_t ph = 0;
    for (long long r = first; r < P.M; r += step) {
        // a wait that ran out is no row: its results are NaNs
        const bool ok = row_is_there(&full[team][s], ph, &gave_up);
        const TX *const row = reinterpret_cast<const TX *>(mine + (size_t)s * R.stage_bytes);
        two_f32 d[P2], s2 = 0, q2 = 0;
        {
            float f[E];
#pragma unroll
            for (int j = 0; j < NV; ++j) read_vector(row, col, j, *reinterpret_cast<float(*)[V]>(f + j * V));
#pragma unroll
            for (int i = 0; i < P2; ++i) {
                d[i] = two(f[2 * i], f[2 * i + 1]);
                s2 = add2(s2, d[i]);
            }
        }
        float sum[1] = {ok ? sum2(s2) : __uint_as_float(0x7FC00000u)};
        if constexpr (TT > 0) team_sum<TT>(sum, red, turn, barrier);
        else team_sum(sum, T, red, turn, barrier);
        // the whole team has its elements: the stage is free
        if (T == 32) __syncwarp();
        if (t == 0 && ok) issue(r + R.stages * step, s);
        const float mean = sum[0] * inv;
        const two_f32 minus = two(-mean, -mean);
#pragma unroll
        for (int i = 0; i < P2; ++i) {
            d[i] = add2(d[i], minus);
            // nothing of what is past the row's end
            if (!col.whole(2 * i / V) && col(2 * i / V) >= C) d[i] = 0;
            q2 = fma2(d[i], d[i], q2);
        }
        float q[1] = {sum2(q2)};
        if constexpr (TT > 0) team_sum<TT>(q, red, turn, barrier);
        else team_sum(q, T, red, turn, barrier);
        const float rstd = rsqrtf(fmaf(q[0], inv, P.eps));
        const two_f32 scale = two(rstd, rstd);
        TY *y = static_cast<TY *>(P.Y) + r * P.ldy;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!col.whole(j) && col(j) >= C) continue;
            float ga[V], be[V], o[V];
            read_param<V>(gammas, P.gamma, col(j), C, 1.0f, ga);
            read_param<V>(betas, P.beta, col(j), C, 0.0f, be);
#pragma unroll
            for (int i = 0; i < V / 2; ++i)
                each(fma2(mul2(d[j * V / 2 + i], scale), two(ga[2 * i], ga[2 * i + 1]), two(be[2 * i], be[2 * i + 1])), o[2 * i], o[2 * i + 1]);
            store(y + col(j), o);
        }
        if (t == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
        if (++s == R.stages) { s = 0; ph ^= 1u; }
    }
    leave_rows(&gave_up);
}

// Rows longer than the registers of a block: the row is read three times, from L2 after the first.  A thread adds its vectors' sums in fp64, so that the
// row's sums are as good as those of shorter rows however many they are (in fp32 rows of 2^22 to 2^27 had 1 / deviation off by 5e-6 to 3.5e-5).
template <typename TX, typename TY, int V>
__global__ void __launch_bounds__(1024) norm_fwd_long_kernel(const __grid_constant__ FwdParams P)
{
    __shared__ __align__(16) float red[2][32][2];
    unsigned int turn = 0;
    const float inv = 1.0f / (float)P.C;
    pdl_begin();
    for (long long r = blockIdx.x; r < P.M; r += gridDim.x) {
        const TX *x = static_cast<const TX *>(P.X) + r * P.ldx;
        float s[1], f[V];
        double total = 0.0;
        for (long long col = (long long)threadIdx.x * V; col < P.C; col += 1024 * V) {
            Vec<TX, V> v;
            v.load(x + col);
            v.get(f);
            float v_sum = f[0];
#pragma unroll
            for (int i = 1; i < V; ++i) v_sum += f[i];
            total += (double)v_sum;
        }
        s[0] = (float)total;
        team_sum(s, 1024, red, turn, 0);
        const float mean = s[0] * inv;
        float q[1];
        total = 0.0;
        for (long long col = (long long)threadIdx.x * V; col < P.C; col += 1024 * V) {
            Vec<TX, V> v;
            v.load(x + col);
            v.get(f);
            float v_sum = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) v_sum = fmaf(f[i] - mean, f[i] - mean, v_sum);
            total += (double)v_sum;
        }
        q[0] = (float)total;
        team_sum(q, 1024, red, turn, 0);
        const float rstd = rsqrtf(fmaf(q[0], inv, P.eps));
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

template <typename TX, typename TY, int V, int E, int TT> int launch_fwd(FwdParams &P, int T, cudaStream_t s)
{
    P.T = T;
    int teams = T > 32 ? 1 : 128 / T;
    // Up to two rows for every team of a block an SM: a launch of that many blocks may start early.  Above, more and smaller blocks balance better.
    const int most = T > kFwdThreads ? 1 : kFwdThreads / T;
    if (P.M <= 2ll * kPdlBlocks * most) {
        teams = (int)std::min<long long>((P.M + kPdlBlocks - 1) / kPdlBlocks, most);
        teams = (teams * T + 31) / 32 * 32 / T;              // whole warps
    }
    const int block = teams * T;
    const long long grid = std::min<long long>((P.M + teams - 1) / teams, 2ll * kPdlBlocks * most >= P.M ? kPdlBlocks : 148ll * 64);
    if (TT > 32 && TT < kFwdThreads && teams > 1)
        TWN_CUDA_OK(twn_launch_small(norm_fwd_kernel<TX, TY, V, E, TT, (TT > 32 && TT < kFwdThreads)>, (int)grid, block, 0, s, P));
    else
        TWN_CUDA_OK(twn_launch_small(norm_fwd_kernel<TX, TY, V, E, TT, false>, (int)grid, block, 0, s, P));
    return TWN_OK;
}
template <typename TX, typename TY, int V, int E, int TT> int launch_fwd_ring(const FwdParams &P, const RingShape &r, const twn_device_info &dev, cudaStream_t s)
{
    static bool done[64] = {false};
    const int rc = allow_ring(norm_fwd_ring_kernel<TX, TY, V, E, TT>, dev.ordinal, done);
    if (rc != TWN_OK) return rc;
    const int grid = (int)std::min<long long>((P.M + r.teams - 1) / r.teams, dev.sm_count);
    TWN_CUDA_OK(twn_launch_small(norm_fwd_ring_kernel<TX, TY, V, E, TT>, grid, r.T * r.teams, r.smem, s, P, r.ring));
    return TWN_OK;
}
template <typename TX, typename TY, int V, int E> bool fwd_ring(FwdParams &P, const twn_device_info &dev, cudaStream_t s, int &rc)
{
    RingShape r;
    if (!ring_shape(r, kFwdRingBytes, P.C, E, fwd_ring_threads<E>(), P.C * sizeof(TX), 0, 2 * sizeof(float) * P.C)) return false;
    P.T = r.T;
    const int filled = P.C == (long long)r.T * E ? r.T : 0;
    if constexpr (E == 64) {
        rc = filled == 32    ? launch_fwd_ring<TX, TY, V, E, 32>(P, r, dev, s)
             : filled == 64  ? launch_fwd_ring<TX, TY, V, E, 64>(P, r, dev, s)
             : filled == 128 ? launch_fwd_ring<TX, TY, V, E, 128>(P, r, dev, s)
             : filled == 256 ? launch_fwd_ring<TX, TY, V, E, 256>(P, r, dev, s)
             : filled == 512 ? launch_fwd_ring<TX, TY, V, E, 512>(P, r, dev, s)
                             : launch_fwd_ring<TX, TY, V, E, 0>(P, r, dev, s);
    } else {
        rc = filled == 32 ? launch_fwd_ring<TX, TY, V, E, 32>(P, r, dev, s) : launch_fwd_ring<TX, TY, V, E, 0>(P, r, dev, s);
    }
    return true;
}
// Rows that the register kernel takes with one block an SM, one or two for a team, it takes faster (two of more than 8192 elements it does not):
// 1030 x 1024 bf16 2.7 us, 4.6 through a ring, 500 x 4096 4.3 and 5.1, 148 x 8000 3.2 and 8.4, 148 x 16384 4.2 and 5.7; 2600 x 1024 6.2 and 4.6.
bool few_rows(const FwdParams &P)
{
    if (P.C > 8192) return P.C <= 16384 && P.M <= kPdlBlocks;
    return P.M <= 2ll * kPdlBlocks * (kFwdThreads / team_for(P.C, 16, 32, 512));
}
template <typename TX, typename TY, int V> int fwd(FwdParams &P, const twn_device_info &dev, cudaStream_t s)
{
    if constexpr (V > 1) {
        int rc = TWN_OK;
        if (P.C > 256 && P.M * P.C >= kRingElements && !few_rows(P) &&
            (P.C <= 512 ? fwd_ring<TX, TY, V, 16>(P, dev, s, rc)
             : P.C <= 1024 ? fwd_ring<TX, TY, V, 32>(P, dev, s, rc)
                           : fwd_ring<TX, TY, V, 64>(P, dev, s, rc)))
            return rc;
    }
    if (P.C <= 32 * 8) return launch_fwd<TX, TY, V, 8, 0>(P, team_for(P.C, 8, 4, 32), s);
    if constexpr (V > 1) {
        if (P.C <= 512) return launch_fwd<TX, TY, V, 16, 32>(P, 32, s);
        if (P.C <= 1024) return launch_fwd<TX, TY, V, 16, 64>(P, 64, s);
        if (P.C <= 2048) return launch_fwd<TX, TY, V, 16, 128>(P, 128, s);
        if (P.C <= 4096) return launch_fwd<TX, TY, V, 16, 256>(P, 256, s);
        if (P.C <= 8192) return launch_fwd<TX, TY, V, 16, 512>(P, 512, s);
        if (P.C <= 16384) return launch_fwd<TX, TY, V, 32, 512>(P, 512, s);
        if (P.C <= 32768) return launch_fwd<TX, TY, V, 32, 1024>(P, 1024, s);
    } else {
        if (P.C <= 512) return launch_fwd<TX, TY, 1, 16, 32>(P, 32, s);
        if (P.C <= 1024) return launch_fwd<TX, TY, 1, 16, 64>(P, 64, s);
        if (P.C <= 2048) return launch_fwd<TX, TY, 1, 16, 128>(P, 128, s);
        if (P.C <= 4096) return launch_fwd<TX, TY, 1, 16, 256>(P, 256, s);
        if (P.C <= 8192) return launch_fwd<TX, TY, 1, 16, 512>(P, 512, s);
        if (P.C <= 16384) return launch_fwd<TX, TY, 1, 16, 1024>(P, 1024, s);
    }
    const int grid = (int)std::min<long long>(P.M, 148 * 2);
    TWN_CUDA_OK(twn_launch_small(norm_fwd_long_kernel<TX, TY, V>, grid, 1024, 0, s, P));
    return TWN_OK;
}
template <typename TX, typename TY> int fwd_any(FwdParams &P, bool vec, const twn_device_info &dev, cudaStream_t s)
{
    constexpr int V = sizeof(TX) == 2 ? 8 : 4;
    return vec ? fwd<TX, TY, V>(P, dev, s) : fwd<TX, TY, 1>(P, dev, s);
}

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
    Places places;
    places.matrix(Y, y_dtype, ldy, M, C, true);
    places.matrix(X, x_dtype, ldx, M, C, false);
    for (const void *p : {(const void *)gamma, (const void *)beta}) places.vector(p, 4 * C, false);
    for (const void *p : {(const void *)mean, (const void *)rstd}) places.vector(p, 4 * M, true);
    TWN_REQUIRE(places.apart(), TWN_ERR_INVALID_ARG);
    twn_device_info dev;
    rc = twn_current_device(&dev);
    if (rc != TWN_OK) return rc;
    FwdParams P = {X, Y, gamma, beta, mean, rstd, ldx, ldy, M, C, (float)eps, 0};
    const int V = x_dtype == TWN_BF16 ? 8 : 4;
    const bool vec = vector_rows(X, x_dtype, ldx, V) && vector_rows(Y, y_dtype, ldy, V) && C % V == 0 && twn_aligned(gamma, 16) &&
                     twn_aligned(beta, 16);
    cudaStream_t s = twn_cu(stream);
    if (x_dtype == TWN_BF16) return y_dtype == TWN_BF16 ? fwd_any<bf16, bf16>(P, vec, dev, s) : fwd_any<bf16, float>(P, vec, dev, s);
    return y_dtype == TWN_BF16 ? fwd_any<float, bf16>(P, vec, dev, s) : fwd_any<float, float>(P, vec, dev, s);
}
