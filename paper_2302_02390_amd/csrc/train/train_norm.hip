// Layer norm of rows and its gradients.
//
//   mu = sum x / n, r = 1 / sqrt(sum (x - mu)^2 / n + eps), h = (x - mu) r, y = h w + b
//   g = dy w, dx = r (g - mean g - h mean(g h)), dw = sum over rows of dy h, db = sum over rows of dy
// The variance is the mean of the centred squares, not a difference of two means, so rows far from zero keep their digits.
#include "train_common.hpp"
#include "train_norm.hpp"
#include "train_plan.hpp"

namespace qsdp_train {
namespace {

// Over a team of TEAM threads: every thread gets the sums. Teams of more than a wave meet in `scratch` (a word for each wave and
// value), in the order of their waves; all teams of the workgroup come here together then.
template <int TEAM, int N>
__device__ __forceinline__ void team_sums(float (&v)[N], float* scratch) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = reduce64(v[i], Add());
    if constexpr (TEAM > 64) {
        constexpr int WAVES = TEAM / 64;
        const int wave = threadIdx.x / 64, lead = wave / WAVES * WAVES;
        __syncthreads();  // what was here before has been read
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) scratch[wave * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = scratch[lead * N + i];
            for (int w = 1; w < WAVES; ++w) v[i] += scratch[(lead + w) * N + i];
        }
    }
}

// ---- forward -------------------------------------------------------------------------------------------------------------
// A team keeps its row in registers between mean, variance and output: one read, one write. It goes on to the row a grid further,
// whose elements are on their way meanwhile; weight and bias stay in a wave's registers. 16384 x 2048 in bf16, 134 MB, takes 28 us or
// 4.7 TB/s (29 in workgroups of one or two teams, 35 with a wave to a row).
template <class X, class Y, int THREADS, int TEAM, int NV>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormParams p) {
    __shared__ float scratch[THREADS / 64];
    constexpr int TEAMS = THREADS / TEAM;
    const int n = (int)p.n, t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    Raw8<X> next[NV];
    auto fetch = [&](uint64_t row) __attribute__((always_inline)) {
        const auto* x = static_cast<const typename X::raw*>(p.x) + row * p.x_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (i * TEAM + t) * 8;
            if (row < p.rows && k < n) next[i].load(x + k, n - k);
            else next[i].none();
        }
    };
    const uint64_t step = (uint64_t)gridDim.x * TEAMS;
    fetch((uint64_t)blockIdx.x * TEAMS + team);
    constexpr bool KEEP = NV <= 2;  // longer rows' come out of the caches
    float w[KEEP ? NV : 1][8], b[KEEP ? NV : 1][8];
    if constexpr (KEEP) {
        Parameters8 of[2][NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (i * TEAM + t) * 8;
            of[0][i].load(p.weight, p.w_dtype, k, n - k);
            of[1][i].load(p.bias, p.w_dtype, k, n - k);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            of[0][i].get(p.weight, p.w_dtype, 1.0f, w[i]);
            of[1][i].get(p.bias, p.w_dtype, 0.0f, b[i]);
        }
    }
    const float count = (float)p.n;
    for (uint64_t base = (uint64_t)blockIdx.x * TEAMS; base < p.rows; base += step) {
        const uint64_t row = base + team;
        float v[NV][8], sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] = next[i].at(e);
                sum[0] += v[i][e];
            }
        if (base + step < p.rows) fetch(row + step);
        team_sums<TEAM>(sum, scratch);
        const float mean = sum[0] / count;
        sum[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (i * TEAM + t) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] = k + e < n ? v[i][e] - mean : 0.0f;
                sum[0] = fmaf(v[i][e], v[i][e], sum[0]);
            }
        }
        team_sums<TEAM>(sum, scratch);
        const float rstd = 1.0f / sqrtf(sum[0] / count + p.eps);
        if (row >= p.rows) continue;
        if (p.stats && t == 0) {
            p.stats[2 * row] = mean;
            p.stats[2 * row + 1] = rstd;
        }
        auto* y = static_cast<typename Y::raw*>(p.y) + row * p.y_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (i * TEAM + t) * 8;
            if (k >= n) continue;
            if constexpr (!KEEP) {
                Parameters8 of[2];
                of[0].load(p.weight, p.w_dtype, k, n - k);
                of[1].load(p.bias, p.w_dtype, k, n - k);
                of[0].get(p.weight, p.w_dtype, 1.0f, w[0]);
                of[1].get(p.bias, p.w_dtype, 0.0f, b[0]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = fmaf(v[i][e] * rstd, w[KEEP ? i : 0][e], b[KEEP ? i : 0][e]);
            store8<Y>(y + k, n - k, v[i]);
        }
    }
}

// Rows that no team holds: read three times.
template <class X, class Y>
__global__ __launch_bounds__(1024) void norm_stream_kernel(NormParams p) {
    __shared__ float scratch[16];
    const int n = (int)p.n;
    const uint64_t row = p.first + blockIdx.x;
    const auto* x = static_cast<const typename X::raw*>(p.x) + row * p.x_stride;
    auto* y = static_cast<typename Y::raw*>(p.y) + row * p.y_stride;
    const float count = (float)p.n;
    float sum[1] = {0.0f};
    Raw8<X> raw;
    for (int k = (int)threadIdx.x * 8; k < n; k += 8192) {
        raw.load(x + k, n - k);
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) part += raw.at(e);
        sum[0] += part;
    }
    team_sums<1024>(sum, scratch);
    const float mean = sum[0] / count;
    sum[0] = 0.0f;
    for (int k = (int)threadIdx.x * 8; k < n; k += 8192) {
        raw.load(x + k, n - k);
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = k + e < n ? raw.at(e) - mean : 0.0f;
            part = fmaf(d, d, part);
        }
        sum[0] += part;
    }
    team_sums<1024>(sum, scratch);
    const float rstd = 1.0f / sqrtf(sum[0] / count + p.eps);
    if (p.stats && threadIdx.x == 0) {
        p.stats[2 * row] = mean;
        p.stats[2 * row + 1] = rstd;
    }
    for (int k = (int)threadIdx.x * 8; k < n; k += 8192) {
        raw.load(x + k, n - k);
        float w[8], b[8], v[8];
        Parameters8 of[2];
        of[0].load(p.weight, p.w_dtype, k, n - k);
        of[1].load(p.bias, p.w_dtype, k, n - k);
        of[0].get(p.weight, p.w_dtype, 1.0f, w);
        of[1].get(p.bias, p.w_dtype, 0.0f, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf((raw.at(e) - mean) * rstd, w[e], b[e]);
        store8<Y>(y + k, n - k, v);
    }
}

// ---- backward ------------------------------------------------------------------------------------------------------------
// Workgroup g takes the rows g, g + G, ... of its teams; a team holds its row of x and dy, and the sums over its rows of dy h
// and dy for its columns, in registers. The teams' sums meet in LDS and are added in their order, the workgroups' in a kernel after
// this one: no atomics, so equal calls give equal bits. Bytes bound long calls: 16384 x 2048 in bf16, 201 MB, 38 us or 5.3 TB/s.
template <class X, class Y, int THREADS, int TEAM, int NV>
__global__ __launch_bounds__(THREADS, THREADS / 256) void norm_backward_kernel(NormBackwardParams p) {
    constexpr int TEAMS = THREADS / TEAM;
    __shared__ float scratch[2 * THREADS / 64];
    __shared__ __attribute__((aligned(16))) f32x4 meet[TEAMS > 1 ? TEAMS : 1][2][TEAMS > 1 ? TEAM : 1][2];  // the teams' sums for dw and db
    const int n = (int)p.n, t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const auto* x = static_cast<const typename X::raw*>(p.x);
    const auto* dy = static_cast<const typename Y::raw*>(p.dy);
    Raw8<X> x_next[NV];
    Raw8<Y> y_next[NV];
    float mean_next = 0.0f, rstd_next = 0.0f;
    auto fetch = [&](uint64_t row) __attribute__((always_inline)) {
        const bool here = row < p.rows;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (i * TEAM + t) * 8;
            if (here && k < n) {
                x_next[i].load(x + row * p.x_stride + k, n - k);
                y_next[i].load(dy + row * p.dy_stride + k, n - k);
            } else {
                x_next[i].none();
                y_next[i].none();
            }
        }
        mean_next = here ? p.stats[2 * row] : 0.0f;
        rstd_next = here ? p.stats[2 * row + 1] : 0.0f;
    };
    const uint64_t step = (uint64_t)gridDim.x * TEAMS;
    const float inverse = 1.0f / (float)p.n;
    fetch((uint64_t)blockIdx.x * TEAMS + team);
    // the weight, as all teams take it, in LDS: in registers it would be a quarter of what a lane has
    __shared__ __attribute__((aligned(16))) f32x4 weight[NV][2][TEAM];
    float dw[NV][8], db[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (team == 0) {
            float w[8];
            Parameters8 of;
            of.load(p.weight, p.w_dtype, (i * TEAM + t) * 8, n - (i * TEAM + t) * 8);
            of.get(p.weight, p.w_dtype, 1.0f, w);
            weight[i][0][t] = f32x4{w[0], w[1], w[2], w[3]};
            weight[i][1][t] = f32x4{w[4], w[5], w[6], w[7]};
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[i][e] = db[i][e] = 0.0f;
    }
    __syncthreads();
    for (uint64_t base = (uint64_t)blockIdx.x * TEAMS; base < p.rows; base += step) {
        const uint64_t row = base + team;
        Raw8<X> xr[NV];
        Raw8<Y> yr[NV];
        const float mean = mean_next, r = rstd_next;
        asm volatile("" ::: "memory");  // the weight is read anew
        float sums[2] = {0.0f, 0.0f};
        // h of an element; past the row's end it meets a dy of zero
        auto centred = [&](int i, int e) __attribute__((always_inline)) { return (xr[i].at(e) - mean) * r; };
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            xr[i] = x_next[i];
            yr[i] = y_next[i];
            const f32x4 w[2] = {weight[i][0][t], weight[i][1][t]};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float h = centred(i, e), y = yr[i].at(e), g = y * w[e / 4][e % 4];
                dw[i][e] = fmaf(y, h, dw[i][e]);
                db[i][e] += y;
                sums[0] += g;
                sums[1] = fmaf(g, h, sums[1]);
            }
        }
        if (base + step < p.rows) fetch(row + step);
        if (!p.dx) continue;
        team_sums<TEAM>(sums, scratch);
        if (row >= p.rows) continue;
        const float c0 = sums[0] * inverse, c1 = sums[1] * inverse;
        auto* dx = static_cast<typename X::raw*>(p.dx) + row * p.dx_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (i * TEAM + t) * 8;
            if (k >= n) continue;
            xr[i].again();  // what is computed of it a second time takes fewer registers than what would be kept
            yr[i].again();
            const f32x4 w[2] = {weight[i][0][t], weight[i][1][t]};
            float d[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = r * (yr[i].at(e) * w[e / 4][e % 4] - fmaf(centred(i, e), c1, c0));
            store8<X>(dx + k, n - k, d);
        }
    }
    if (!p.partial) return;
    float* to = p.partial + (uint64_t)blockIdx.x * 2 * p.n;
    if constexpr (TEAMS > 1) {
        static_assert(NV == 1, "a piece of a row to a thread");
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            meet[team][0][t][h] = f32x4{dw[0][4 * h], dw[0][4 * h + 1], dw[0][4 * h + 2], dw[0][4 * h + 3]};
            meet[team][1][t][h] = f32x4{db[0][4 * h], db[0][4 * h + 1], db[0][4 * h + 2], db[0][4 * h + 3]};
        }
        __syncthreads();
#pragma unroll
        for (int c = threadIdx.x; c < 16 * TEAM; c += THREADS) {
            const float* from = reinterpret_cast<const float*>(meet) + c;
            float sum = from[0];
#pragma unroll
            for (int other = 1; other < TEAMS; ++other) sum += from[other * 16 * TEAM];
            const int of = c / (8 * TEAM), k = c % (8 * TEAM);
            if (k < n) to[of * p.n + k] = sum;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (i * TEAM + t) * 8;
            if (k >= n) continue;
            store8<F32>(to + k, n - k, dw[i]);
            store8<F32>(to + p.n + k, n - k, db[i]);
        }
    }
}

// Rows that no team holds: dx of a row by a workgroup, which reads it twice ...
template <class X, class Y>
__global__ __launch_bounds__(1024) void norm_rows_backward_kernel(NormBackwardParams p, uint64_t first) {
    __shared__ float scratch[32];
    const int n = (int)p.n;
    const uint64_t row = first + blockIdx.x;
    const auto* x = static_cast<const typename X::raw*>(p.x) + row * p.x_stride;
    const auto* dy = static_cast<const typename Y::raw*>(p.dy) + row * p.dy_stride;
    auto* dx = static_cast<typename X::raw*>(p.dx) + row * p.dx_stride;
    const float mean = p.stats[2 * row], r = p.stats[2 * row + 1], inverse = 1.0f / (float)p.n;
    float sums[2] = {0.0f, 0.0f};
    Raw8<X> xr;
    Raw8<Y> yr;
    for (int k = (int)threadIdx.x * 8; k < n; k += 8192) {
        xr.load(x + k, n - k);
        yr.load(dy + k, n - k);
        float w[8], part[2] = {0.0f, 0.0f};
        Parameters8 of;
        of.load(p.weight, p.w_dtype, k, n - k);
        of.get(p.weight, p.w_dtype, 1.0f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float g = yr.at(e) * w[e], h = k + e < n ? (xr.at(e) - mean) * r : 0.0f;
            part[0] += g;
            part[1] = fmaf(g, h, part[1]);
        }
        sums[0] += part[0];
        sums[1] += part[1];
    }
    team_sums<1024>(sums, scratch);
    const float c0 = sums[0] * inverse, c1 = sums[1] * inverse;
    for (int k = (int)threadIdx.x * 8; k < n; k += 8192) {
        xr.load(x + k, n - k);
        yr.load(dy + k, n - k);
        float w[8], d[8];
        Parameters8 of;
        of.load(p.weight, p.w_dtype, k, n - k);
        of.get(p.weight, p.w_dtype, 1.0f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = r * (yr.at(e) * w[e] - fmaf((xr.at(e) - mean) * r, c1, c0));
        store8<X>(dx + k, n - k, d);
    }
}

// ... and the sums of 2048 columns over a run of rows by another.
template <class X, class Y>
__global__ __launch_bounds__(256) void norm_columns_backward_kernel(NormBackwardParams p, uint64_t groups) {
    const auto* x = static_cast<const typename X::raw*>(p.x);
    const auto* dy = static_cast<const typename Y::raw*>(p.dy);
    const int n = (int)p.n, k = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 8;
    if (k >= n) return;
    float dw[8], db[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] = db[e] = 0.0f;
    for (uint64_t row = blockIdx.y; row < p.rows; row += groups) {
        Raw8<X> xr;
        Raw8<Y> yr;
        xr.load(x + row * p.x_stride + k, n - k);
        yr.load(dy + row * p.dy_stride + k, n - k);
        const float mean = p.stats[2 * row], r = p.stats[2 * row + 1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = yr.at(e);
            dw[e] = fmaf(y, k + e < n ? (xr.at(e) - mean) * r : 0.0f, dw[e]);
            db[e] += y;
        }
    }
    float* to = p.partial + (uint64_t)blockIdx.y * 2 * p.n;
    store8<F32>(to + k, n - k, dw);
    store8<F32>(to + p.n + k, n - k, db);
}

// Sums of the workgroups' partial sums: 16 columns to a workgroup, whose 16 groups of threads take every sixteenth partial, sixteen of
// them on their way at a time.
__global__ __launch_bounds__(256) void norm_total_kernel(const float* partial, uint64_t workgroups, uint64_t n, float* dw,
                                                        float* db, bool accumulate) {
    __shared__ float sums[16][17];
    const uint64_t at = (uint64_t)blockIdx.x * 16 + threadIdx.x % 16;  // of the 2 n columns
    const int part = threadIdx.x / 16;
    float sum = 0.0f;
    if (at < 2 * n) {
        for (uint64_t g = part; g < workgroups; g += 16 * 16) {
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = g + i * 16 < workgroups ? partial[(g + i * 16) * 2 * n + at] : 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += v[i];
        }
    }
    sums[part][threadIdx.x % 16] = sum;
    __syncthreads();
    if (part || at >= 2 * n) return;
    for (int i = 1; i < 16; ++i) sum += sums[i][threadIdx.x];
    float* to = at < n ? dw : db;
    if (!to) return;
    to += at < n ? at : at - n;
    *to = accumulate ? *to + sum : sum;
}

}  // namespace

template <class X, class Y, int THREADS, int TEAM, int NV>
static hipError_t launch_team(const NormParams& p, hipStream_t s) {
    constexpr uint64_t EACH = THREADS / TEAM, MOST = 256 * (1024 / THREADS);  // 16 waves to a compute unit
    const uint64_t need = (p.rows + EACH - 1) / EACH;
    hipLaunchKernelGGL((norm_kernel<X, Y, THREADS, TEAM, NV>), dim3((unsigned)(need < MOST ? need : MOST)), dim3(THREADS), 0, s, p);
    return hipGetLastError();
}

template <class X, class Y>
static hipError_t launch_norm_of(NormParams p, hipStream_t s) {
    switch (choose_norm(p.rows, p.n)) {
        case NormTeam::T64: return launch_team<X, Y, 256, 64, 1>(p, s);
        case NormTeam::T64_2: return launch_team<X, Y, 512, 64, 2>(p, s);
        case NormTeam::T128_2: return launch_team<X, Y, 512, 128, 2>(p, s);
        case NormTeam::T256_2: return launch_team<X, Y, 512, 256, 2>(p, s);
        case NormTeam::T512_2: return launch_team<X, Y, 512, 512, 2>(p, s);
        case NormTeam::T1024_2: return launch_team<X, Y, 1024, 1024, 2>(p, s);
        case NormTeam::T1024_4: return launch_team<X, Y, 1024, 1024, 4>(p, s);
        case NormTeam::SHORT: return launch_team<X, Y, 256, 256, 1>(p, s);
        case NormTeam::STREAM: break;
    }
    for (p.first = 0; p.first < p.rows; p.first += kMaxGrid) {
        const uint64_t left = p.rows - p.first;
        hipLaunchKernelGGL((norm_stream_kernel<X, Y>), dim3((unsigned)(left < kMaxGrid ? left : kMaxGrid)), dim3(1024), 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// f with null pointers to the formats of x and of y (that of x, or any for binary32).
template <class F>
static hipError_t by_formats(qsdp_dtype x, qsdp_dtype y, F f) {
    if (x == QSDP_BF16) return f((BF16*)nullptr, (BF16*)nullptr);
    if (x == QSDP_F16) return f((F16*)nullptr, (F16*)nullptr);
    if (y == QSDP_BF16) return f((F32*)nullptr, (BF16*)nullptr);
    if (y == QSDP_F16) return f((F32*)nullptr, (F16*)nullptr);
    return f((F32*)nullptr, (F32*)nullptr);
}

hipError_t launch_norm(qsdp_dtype x, qsdp_dtype y, NormParams p, hipStream_t s) {
    return by_formats(x, y, [&](auto* a, auto* b) {
        return launch_norm_of<std::remove_pointer_t<decltype(a)>, std::remove_pointer_t<decltype(b)>>(p, s);
    });
}

template <class X, class Y, int THREADS, int TEAM, int NV>
static hipError_t launch_backward_team(const NormBackwardParams& p, hipStream_t s) {
    hipLaunchKernelGGL((norm_backward_kernel<X, Y, THREADS, TEAM, NV>), dim3((unsigned)norm_workgroups(p.rows, p.n)), dim3(THREADS), 0,
                       s, p);
    return hipGetLastError();
}

template <class X, class Y>
static hipError_t launch_norm_backward_of(const NormBackwardParams& p, hipStream_t s) {
    switch (choose_norm_backward(p.n)) {
        case NormBackwardTeam::T64: return launch_backward_team<X, Y, kNormThreads, 64, 1>(p, s);
        case NormBackwardTeam::T128: return launch_backward_team<X, Y, kNormThreads, 128, 1>(p, s);
        case NormBackwardTeam::T256: return launch_backward_team<X, Y, kNormThreads, 256, 1>(p, s);
        case NormBackwardTeam::T512: return launch_backward_team<X, Y, kNormThreads, 512, 1>(p, s);
        case NormBackwardTeam::T1024: return launch_backward_team<X, Y, kNormThreads, 1024, 1>(p, s);
        case NormBackwardTeam::T512_4: return launch_backward_team<X, Y, 512, 512, 4>(p, s);
        case NormBackwardTeam::STREAM: break;
    }
    // the sums first: dx may overwrite what they read
    if (p.partial) {
        const uint64_t groups = norm_workgroups(p.rows, p.n);
        hipLaunchKernelGGL((norm_columns_backward_kernel<X, Y>), dim3((unsigned)((p.n + 2047) / 2048), (unsigned)groups), dim3(256),
                           0, s, p, groups);
    }
    if (p.dx)
        for (uint64_t first = 0; first < p.rows; first += kMaxGrid) {
            const uint64_t left = p.rows - first;
            hipLaunchKernelGGL((norm_rows_backward_kernel<X, Y>), dim3((unsigned)(left < kMaxGrid ? left : kMaxGrid)), dim3(1024),
                               0, s, p, first);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    return hipGetLastError();
}

hipError_t launch_norm_backward(qsdp_dtype x, qsdp_dtype y, const NormBackwardParams& p, float* dw, float* db, bool accumulate,
                                hipStream_t s) {
    if (p.rows == 0) {  // sums of nothing
        hipLaunchKernelGGL(norm_total_kernel, dim3((unsigned)((2 * p.n + 15) / 16)), dim3(256), 0, s, nullptr, 0, p.n, dw, db, false);
        return hipGetLastError();
    }
    const hipError_t e = by_formats(x, y, [&](auto* a, auto* b) {
        return launch_norm_backward_of<std::remove_pointer_t<decltype(a)>, std::remove_pointer_t<decltype(b)>>(p, s);
    });
    if (e != hipSuccess || !p.partial) return e;
    hipLaunchKernelGGL(norm_total_kernel, dim3((unsigned)((2 * p.n + 15) / 16)), dim3(256), 0, s, p.partial,
                       norm_workgroups(p.rows, p.n), p.n, dw, db, accumulate);
    return hipGetLastError();
}

}  // namespace qsdp_train
