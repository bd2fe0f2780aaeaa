// Group norm over channels-last positions, with an activation, forward and backward, and the sums over the samples of the scale's and the
// shift's gradients (Alg. 1, first two lines of the loop body, for those two vectors).  x is [B, P, C], C = G groups of w channels; of
// sample z and group q, over its M = P w elements:
//   forward   mean = sum x / M,  rstd = 1 / sqrt(sum (x - mean)^2 / M + eps),  xhat = (x - mean) rstd,  y = act(gamma xhat + beta)
//   backward  e = dy act'(gamma xhat + beta),  d = e gamma,  dx = rstd (d - sum d / M - xhat sum (d xhat) / M)
//             sample z's gradients  G_z = sum_p e xhat  and  H_z = sum_p e (by channel);  g = c sum_z G_z,  s = c^2 sum_z G_z^2, H likewise
// Everything is float32 between the loads and the stores.  A group's two sums of the backward pass are those of its channels' G_z and
// H_z, weighted by gamma, so nothing is formed twice.
//
// Bound by memory.  Where a sample's channels of a few whole groups fit into a workgroup's registers it reads them once (k_group_norm,
// k_group_norm_backward); larger ones are read twice: by channel and chunk of positions for the sums, which belong to no group yet, and
// once the groups' are joined for the result.  No atomics: results do not depend on scheduling.
#include <algorithm>

#include "vgc_columns.h"
#include "vgc_epilogue.h"

namespace vgc {

struct GroupNormArgs {
    const void *x, *dy;
    const float *gamma, *beta, *mean, *rstd;                 // (mean, rstd: of the passes that read them)
    float *mean_out, *rstd_out;
    void* out;
    float* chunk_sums;        // [sample][chunk][2][C]
    float* sums;              // backward: [sample][G_z, H_z][C]
    float* group_sums;        // backward: [sample][G][sum d / M, sum d xhat / M]
    uint32_t B, P, C, G, w, act;
    float eps;
    uint32_t lanes, blocks, chunks, rows;                    // of a piece row; blocks of columns; chunks of a sample, positions each
    uint32_t groups, slabs;                                  // whole groups a workgroup takes, workgroups a sample
};

// gamma xhat + beta, rounded after each operation in both passes: relu's slope is decided by the sign that the forward pass saw, which with one
// rounding less would be another once in some 10^8 elements.
__device__ __forceinline__ float scaled(float xhat, float gamma, float beta) { return xhat * gamma + beta; }

__device__ __forceinline__ uint32_t at_most(uint32_t a, uint32_t b) { return a < b ? a : b; }

// Sums of chan over whole groups of w channels, a wave a group.  Ends with a barrier.
template <typename Weight>
__device__ __forceinline__ void sums_of_groups(const float* chan, uint32_t w, uint32_t groups, float* grp, Weight weight) {
    const uint32_t lane = threadIdx.x & 63u, waves = blockDim.x / 64u;
    for (uint32_t q = threadIdx.x >> 6; q < groups; q += waves) {
        float sum = 0.f;
        for (uint32_t c = lane; c < w; c += 64u) sum += weight(q * w + c) * chan[q * w + c];
        sum = wave_sum(sum);
        if (lane == 0) grp[q] = sum;
    }
    __syncthreads();
}

// ---- a sample's whole groups in one workgroup ---------------------------------------------------------------------------------
// kNV rows of a team are held as they are in memory.
constexpr uint32_t kMostThreads = 512, kMostSlab = 512;      // threads, channels

template <typename T, int kNV>
__global__ __launch_bounds__(kMostThreads) void k_group_norm(GroupNormArgs A) {
    __shared__ float sh[kMostThreads * 8], part[kMostThreads], chan[kMostSlab], grp[64];
    const uint32_t b = blockIdx.x / A.slabs, slab = blockIdx.x - b * A.slabs, q0 = slab * A.groups, groups = min(A.groups, A.G - q0);
    const uint32_t lane = threadIdx.x % A.lanes, team = threadIdx.x / A.lanes, teams = blockDim.x / A.lanes;
    const uint32_t c0 = q0 * A.w, width = groups * A.w, own = lane * 8u;
    const int n = (int)width - (int)own;                     // channels of this lane that exist: all for 8 or more
    const uint64_t rows = (uint64_t)A.B * A.P;
    const T* x = static_cast<const T*>(A.x) + (uint64_t)b * A.P * A.C + c0 + own;
    Raw8<T> raw[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        const uint32_t p = team + i * teams;
        raw[i] = load8(x + (uint64_t)p * A.C, p < A.P ? n : 0, rows_at_end((uint64_t)b * A.P + p, rows));
    }
    uint32_t of[8];                                          // group of a channel
#pragma unroll
    for (int k = 0; k < 8; ++k) of[k] = k < n ? (own + k) / A.w : 0u;
    float ga[8], be[8];
    widen8(load8(A.gamma + c0 + own, n), ga);
    widen8(load8(A.beta + c0 + own, n), be);
    const float inv = 1.0f / ((float)A.P * (float)A.w);
    auto one = [](uint32_t) { return 1.f; };
    float f[8], v[8] = {};
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        clip8(raw[i], n);
        widen8(raw[i], f);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += f[k];
    }
    channel_sums(v, A.lanes, sh, part, chan);
    sums_of_groups(chan, A.w, groups, grp, one);
    float mean[8], rstd[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) { mean[k] = grp[of[k]] * inv; v[k] = 0.f; }
    const float own_mean = threadIdx.x < groups ? grp[threadIdx.x] * inv : 0.f;
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        widen8(raw[i], f);
        if (team + i * teams < A.P)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float d = k < n ? f[k] - mean[k] : 0.f;
                v[k] = __builtin_fmaf(d, d, v[k]);
            }
    }
    channel_sums(v, A.lanes, sh, part, chan);
    sums_of_groups(chan, A.w, groups, grp, one);
#pragma unroll
    for (int k = 0; k < 8; ++k) rstd[k] = 1.0f / sqrtf(grp[of[k]] * inv + A.eps);
    if (threadIdx.x < groups) {
        A.mean_out[(uint64_t)b * A.G + q0 + threadIdx.x] = own_mean;
        A.rstd_out[(uint64_t)b * A.G + q0 + threadIdx.x] = 1.0f / sqrtf(grp[threadIdx.x] * inv + A.eps);
    }
    T* y = static_cast<T*>(A.out) + (uint64_t)b * A.P * A.C + c0 + own;
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        const uint32_t p = team + i * teams;
        if (p >= A.P || n <= 0) continue;
        widen8(raw[i], f);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = scaled((f[k] - mean[k]) * rstd[k], ga[k], be[k]);
        apply_act((int)A.act, f);
        store8(y + (uint64_t)p * A.C, f, n);
    }
}

// The groups' mean, rstd, gamma and beta for a lane's channels c0 .. (n of them).
struct Channels { float mean[8], rstd[8], gamma[8], beta[8]; };
__device__ __forceinline__ void channels_of(const GroupNormArgs& A, uint32_t b, uint32_t c0, int n, Channels& K) {
    widen8(load8(A.gamma + c0, n), K.gamma);
    widen8(load8(A.beta + c0, n), K.beta);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        K.mean[k] = K.rstd[k] = 0.f;
        if (k >= n) continue;
        const uint64_t at = (uint64_t)b * A.G + (c0 + k) / A.w;
        K.mean[k] = A.mean[at];
        K.rstd[k] = A.rstd[at];
    }
}
// d becomes e = dy act'(gamma xhat + beta), x xhat.
__device__ __forceinline__ void through_act(const GroupNormArgs& A, const Channels& K, float (&x)[8], float (&d)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = (x[k] - K.mean[k]) * K.rstd[k];
    if (A.act == VGC_ACT_NONE) return;
    float t[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) t[k] = scaled(x[k], K.gamma[k], K.beta[k]);
    apply_slope((int)A.act, t, d);
}

template <typename T, int kNV>
__global__ __launch_bounds__(kMostThreads) void k_group_norm_backward(GroupNormArgs A) {
    __shared__ float sh[kMostThreads * 8], part[kMostThreads], chan[2][kMostSlab], grp[2][64];
    const uint32_t b = blockIdx.x / A.slabs, slab = blockIdx.x - b * A.slabs, q0 = slab * A.groups, groups = min(A.groups, A.G - q0);
    const uint32_t lane = threadIdx.x % A.lanes, team = threadIdx.x / A.lanes, teams = blockDim.x / A.lanes;
    const uint32_t c0 = q0 * A.w, width = groups * A.w, own = lane * 8u;
    const int n = (int)width - (int)own;
    const uint64_t rows = (uint64_t)A.B * A.P, at = (uint64_t)b * A.P * A.C + c0 + own;
    Raw8<T> rx[kNV], rd[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        const uint32_t p = team + i * teams;
        const int m = p < A.P ? n : 0;
        rx[i] = load8(static_cast<const T*>(A.x) + at + (uint64_t)p * A.C, m, rows_at_end((uint64_t)b * A.P + p, rows));
        rd[i] = load8(static_cast<const T*>(A.dy) + at + (uint64_t)p * A.C, m, rows_at_end((uint64_t)b * A.P + p, rows));
    }
    Channels K;
    channels_of(A, b, c0 + own, n, K);
    float x[8], d[8], vg[8] = {}, vh[8] = {};
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        if (team + i * teams >= A.P) continue;
        clip8(rd[i], n);
        clip8(rx[i], n);
        widen8(rx[i], x);
        widen8(rd[i], d);
        through_act(A, K, x, d);
#pragma unroll
        for (int k = 0; k < 8; ++k) { vg[k] = __builtin_fmaf(d[k], x[k], vg[k]); vh[k] += d[k]; }
    }
    channel_sums(vg, A.lanes, sh, part, chan[0]);
    channel_sums(vh, A.lanes, sh, part, chan[1]);
    const float* gamma = A.gamma + c0;
    sums_of_groups(chan[1], A.w, groups, grp[0], [&](uint32_t c) { return gamma[c]; });
    sums_of_groups(chan[0], A.w, groups, grp[1], [&](uint32_t c) { return gamma[c]; });
    for (uint32_t c = threadIdx.x; c < 2u * width; c += blockDim.x) {
        const uint32_t v = c >= width, ch = c - v * width;
        A.sums[((uint64_t)b * 2u + v) * A.C + c0 + ch] = chan[v][ch];
    }
    if (n <= 0) return;
    const float inv = 1.0f / ((float)A.P * (float)A.w);
    float m1[8], m2[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t q = k < n ? (own + k) / A.w : 0u;
        m1[k] = grp[0][q] * inv;
        m2[k] = grp[1][q] * inv;
    }
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        const uint32_t p = team + i * teams;
        if (p >= A.P) continue;
        widen8(rx[i], x);
        widen8(rd[i], d);
        through_act(A, K, x, d);
#pragma unroll
        for (int k = 0; k < 8; ++k) d[k] = K.rstd[k] * __builtin_fmaf(-x[k], m2[k], __builtin_fmaf(d[k], K.gamma[k], -m1[k]));
        store8(static_cast<T*>(A.out) + at + (uint64_t)p * A.C, d, n);
    }
}

// ---- samples beyond that: sums by channel and chunk, then the result ------------------------------------------------------------
// Workgroup (sample, block of columns, chunk of positions): teams take the chunk's rows in turn, kRows of them in flight.
struct Place { uint32_t b, chunk, c0, team, teams, p0, p1; int n; };
__device__ __forceinline__ Place place_of(const GroupNormArgs& A) {
    Place L;
    const uint32_t per = A.blocks * A.chunks, rest = blockIdx.x % per, block = rest % A.blocks;
    L.b = blockIdx.x / per;
    L.chunk = rest / A.blocks;
    L.c0 = (block * A.lanes + threadIdx.x % A.lanes) * 8u;
    L.team = threadIdx.x / A.lanes;
    L.teams = blockDim.x / A.lanes;
    L.p0 = L.chunk * A.rows;
    L.p1 = min(L.p0 + A.rows, A.P);
    L.n = (int)A.C - (int)L.c0;
    return L;
}
// Mean and sum of squares about it, by channel.  A lane's sums are relative to the mean of its first kRows rows: what the sum of
// squares then loses to the difference of that mean and its whole mean is at most the share of those rows, whatever the values.  Lanes are joined as
// (count, mean, squares), so that a large mean costs no digits.
constexpr int kRows = 4;
template <typename T>
__global__ __launch_bounds__(256) void k_group_norm_moments(GroupNormArgs A) {
    __shared__ float sm[2048], sq[2048], pm[256], pq[256];
    const Place L = place_of(A);
    const uint64_t rows = (uint64_t)A.B * A.P;
    const T* x = static_cast<const T*>(A.x) + (uint64_t)L.b * A.P * A.C + L.c0;
    Raw8<T> raw[kRows];
    auto request = [&](uint32_t p) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint32_t r = p + i * L.teams;
            raw[i] = load8(x + (uint64_t)r * A.C, r < L.p1 ? L.n : 0, rows_at_end((uint64_t)L.b * A.P + r, rows));
        }
    };
    float base[8] = {}, s1[8] = {}, s2[8] = {}, f[8];
    const uint32_t count = rows_of_team(L.p1 - L.p0, L.team, L.teams), first = at_most(count, kRows);
    uint32_t p = L.p0 + L.team;
    request(p);
    if (first != 0u) {
        const float inv = 1.0f / (float)first;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            widen8(raw[i], f);                               // (zeros past the chunk's end)
#pragma unroll
            for (int k = 0; k < 8; ++k) base[k] += f[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) base[k] *= inv;
    }
    for (; p < L.p1; p += kRows * L.teams) {
        Raw8<T> now[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) now[i] = raw[i];
        if (p + kRows * L.teams < L.p1) request(p + kRows * L.teams);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (p + i * L.teams >= L.p1) continue;
            widen8(now[i], f);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float d = f[k] - base[k];
                s1[k] += d;
                s2[k] = __builtin_fmaf(d, d, s2[k]);
            }
        }
    }
    const float inv = count ? 1.0f / (float)count : 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float m = s1[k] * inv;
        sm[threadIdx.x * 8u + k] = base[k] + m;
        sq[threadIdx.x * 8u + k] = fmaxf(__builtin_fmaf(-s1[k], m, s2[k]), 0.f);
    }
    __syncthreads();
    // eight teams a thread, then the threads of a channel
    const uint32_t S = A.lanes * 8u, c = threadIdx.x % S, sub = threadIdx.x / S, subs = 256u / S, rows_here = L.p1 - L.p0;
    float total = 0.f, mean = 0.f, squares = 0.f;
    for (uint32_t t = 0; t < 8u; ++t) {
        const float m = (float)rows_of_team(rows_here, sub * 8u + t, L.teams);
        total += m;
        mean = __builtin_fmaf(m, sm[(sub * 8u + t) * S + c], mean);
    }
    if (total > 0.f) mean /= total;
    for (uint32_t t = 0; t < 8u; ++t) {
        const float m = (float)rows_of_team(rows_here, sub * 8u + t, L.teams), d = sm[(sub * 8u + t) * S + c] - mean;
        if (m > 0.f) squares += __builtin_fmaf(m * d, d, sq[(sub * 8u + t) * S + c]);
    }
    if (subs > 1u) {
        pm[threadIdx.x] = mean;
        pq[threadIdx.x] = squares;
        __syncthreads();
        if (threadIdx.x >= S) return;
        auto rows_of_sub = [&](uint32_t q) {
            uint32_t r = 0;
            for (uint32_t t = 0; t < 8u; ++t) r += rows_of_team(rows_here, q * 8u + t, L.teams);
            return (float)r;
        };
        mean = squares = 0.f;
        for (uint32_t q = 0; q < subs; ++q) mean = __builtin_fmaf(rows_of_sub(q), pm[q * S + c], mean);
        mean /= (float)rows_here;
        for (uint32_t q = 0; q < subs; ++q) {
            const float m = rows_of_sub(q), d = pm[q * S + c] - mean;
            if (m > 0.f) squares += __builtin_fmaf(m * d, d, pq[q * S + c]);
        }
    }
    const uint32_t col = L.c0 - (threadIdx.x % A.lanes) * 8u + c;          // of the block's columns
    if (col >= A.C) return;
    float* out = A.chunk_sums + ((uint64_t)L.b * A.chunks + L.chunk) * 2u * A.C + col;
    out[0] = mean;
    out[A.C] = squares;
}

__device__ __forceinline__ double wave_sum_double(double x) {
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// A group's moments from those of its channels and chunks; in 64 bits, so that mean^2 may be subtracted.
__global__ __launch_bounds__(256) void k_group_norm_join(GroupNormArgs A) {
    __shared__ double sh[2][4];
    const uint32_t b = blockIdx.x / A.G, q = blockIdx.x - b * A.G, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const float* in = A.chunk_sums + (uint64_t)b * A.chunks * 2u * A.C + q * A.w;
    double s1 = 0., s2 = 0.;
    for (uint32_t e = threadIdx.x; e < A.chunks * A.w; e += blockDim.x) {
        const uint32_t chunk = e / A.w, c = e - chunk * A.w;
        const double m = (double)(min((chunk + 1u) * A.rows, A.P) - chunk * A.rows), mean = in[(uint64_t)chunk * 2u * A.C + c];
        s1 += m * mean;
        s2 += m * mean * mean + (double)in[((uint64_t)chunk * 2u + 1u) * A.C + c];
    }
    s1 = wave_sum_double(s1);
    s2 = wave_sum_double(s2);
    if (lane == 0) { sh[0][wave] = s1; sh[1][wave] = s2; }
    __syncthreads();
    if (threadIdx.x != 0) return;
    s1 = s2 = 0.;
    for (uint32_t v = 0; v < blockDim.x / 64u; ++v) { s1 += sh[0][v]; s2 += sh[1][v]; }
    const double M = (double)A.P * A.w, mean = s1 / M, var = s2 / M - mean * mean;
    A.mean_out[blockIdx.x] = (float)mean;
    A.rstd_out[blockIdx.x] = (float)(1.0 / sqrt((var < 0. ? 0. : var) + (double)A.eps));   // (a NaN stays one)
}

template <typename T>
__global__ __launch_bounds__(256) void k_group_norm_apply(GroupNormArgs A) {
    const Place L = place_of(A);
    if (L.n <= 0) return;
    const uint64_t rows = (uint64_t)A.B * A.P, at = (uint64_t)L.b * A.P * A.C + L.c0;
    const T* x = static_cast<const T*>(A.x) + at;
    T* y = static_cast<T*>(A.out) + at;
    Raw8<T> raw[kRows];
    auto request = [&](uint32_t p) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint32_t r = p + i * L.teams;
            raw[i] = load8(x + (uint64_t)r * A.C, r < L.p1 ? L.n : 0, rows_at_end((uint64_t)L.b * A.P + r, rows));
        }
    };
    uint32_t p = L.p0 + L.team;
    request(p);
    Channels K;
    channels_of(A, L.b, L.c0, L.n, K);
    for (; p < L.p1; p += kRows * L.teams) {
        Raw8<T> now[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) now[i] = raw[i];
        if (p + kRows * L.teams < L.p1) request(p + kRows * L.teams);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint32_t r = p + i * L.teams;
            if (r >= L.p1) continue;
            float f[8];
            widen8(now[i], f);
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = scaled((f[k] - K.mean[k]) * K.rstd[k], K.gamma[k], K.beta[k]);
            apply_act((int)A.act, f);
            store8(y + (uint64_t)r * A.C, f, L.n);
        }
    }
}

// kSums: G_z and H_z of the chunk; else dx.
template <typename T, bool kSums>
__global__ __launch_bounds__(256) void k_group_norm_backward_rows(GroupNormArgs A) {
    __shared__ float sh[kSums ? 2048 : 1], part[kSums ? 256 : 1], chan[kSums ? 256 : 1];
    const Place L = place_of(A);
    if (!kSums && L.n <= 0) return;
    const uint64_t rows = (uint64_t)A.B * A.P, at = (uint64_t)L.b * A.P * A.C + L.c0;
    constexpr int kR = kRows / 2;
    Raw8<T> rx[kR], rd[kR];
    auto request = [&](uint32_t p) {
#pragma unroll
        for (int i = 0; i < kR; ++i) {
            const uint32_t r = p + i * L.teams;
            const bool at_end = rows_at_end((uint64_t)L.b * A.P + r, rows);
            rx[i] = load8(static_cast<const T*>(A.x) + at + (uint64_t)r * A.C, r < L.p1 ? L.n : 0, at_end);
            rd[i] = load8(static_cast<const T*>(A.dy) + at + (uint64_t)r * A.C, r < L.p1 ? L.n : 0, at_end);
        }
    };
    uint32_t p = L.p0 + L.team;
    request(p);
    Channels K;
    channels_of(A, L.b, L.c0, L.n, K);
    float m1[8] = {}, m2[8] = {};
    if (!kSums)
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < L.n) {
                const float* g = A.group_sums + ((uint64_t)L.b * A.G + (L.c0 + k) / A.w) * 2u;
                m1[k] = g[0];
                m2[k] = g[1];
            }
    float vg[8] = {}, vh[8] = {};
    for (; p < L.p1; p += kR * L.teams) {
        Raw8<T> nx[kR], nd[kR];
#pragma unroll
        for (int i = 0; i < kR; ++i) { nx[i] = rx[i]; nd[i] = rd[i]; }
        if (p + kR * L.teams < L.p1) request(p + kR * L.teams);
#pragma unroll
        for (int i = 0; i < kR; ++i) {
            const uint32_t r = p + i * L.teams;
            if (r >= L.p1) continue;
            float x[8], d[8];
            clip8(nx[i], L.n);
            clip8(nd[i], L.n);
            widen8(nx[i], x);
            widen8(nd[i], d);
            through_act(A, K, x, d);
            if (kSums) {
#pragma unroll
                for (int k = 0; k < 8; ++k) { vg[k] = __builtin_fmaf(d[k], x[k], vg[k]); vh[k] += d[k]; }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) d[k] = K.rstd[k] * __builtin_fmaf(-x[k], m2[k], __builtin_fmaf(d[k], K.gamma[k], -m1[k]));
                store8(static_cast<T*>(A.out) + at + (uint64_t)r * A.C, d, L.n);
            }
        }
    }
    if (!kSums) return;
    const uint32_t first = L.c0 - (threadIdx.x % A.lanes) * 8u, c = first + threadIdx.x;
    float* out = A.chunk_sums + ((uint64_t)L.b * A.chunks + L.chunk) * 2u * A.C;
    channel_sums(vg, A.lanes, sh, part, chan);
    if (threadIdx.x < A.lanes * 8u && c < A.C) out[c] = chan[threadIdx.x];
    __syncthreads();
    channel_sums(vh, A.lanes, sh, part, chan);
    if (threadIdx.x < A.lanes * 8u && c < A.C) out[A.C + c] = chan[threadIdx.x];
}

// G_z and H_z of a group's channels from their chunks, and the group's two sums.
__global__ __launch_bounds__(256) void k_group_norm_backward_join(GroupNormArgs A) {
    __shared__ float sh[2][256], total[2][4];
    const uint32_t b = blockIdx.x / A.G, q = blockIdx.x - b * A.G;
    uint32_t wp = 1;
    while (wp < A.w && wp < 256u) wp *= 2u;
    const uint32_t ch = threadIdx.x % wp, sub = threadIdx.x / wp, subs = 256u / wp;
    float m1 = 0.f, m2 = 0.f;
    for (uint32_t c0 = 0; c0 < A.w; c0 += wp) {
        const uint32_t c = c0 + ch, col = q * A.w + c;
        float g = 0.f, h = 0.f;
        if (c < A.w) {
            const float* in = A.chunk_sums + (uint64_t)b * A.chunks * 2u * A.C + col;
#pragma unroll 4
            for (uint32_t k = sub; k < A.chunks; k += subs) { g += in[(uint64_t)k * 2u * A.C]; h += in[((uint64_t)k * 2u + 1u) * A.C]; }
        }
        sh[0][threadIdx.x] = g;
        sh[1][threadIdx.x] = h;
        __syncthreads();
        if (sub == 0u && c < A.w) {
            for (uint32_t s = 1; s < subs; ++s) { g += sh[0][s * wp + ch]; h += sh[1][s * wp + ch]; }
            A.sums[(uint64_t)b * 2u * A.C + col] = g;
            A.sums[((uint64_t)b * 2u + 1u) * A.C + col] = h;
            const float gamma = A.gamma[col];
            m1 = __builtin_fmaf(gamma, h, m1);
            m2 = __builtin_fmaf(gamma, g, m2);
        }
        __syncthreads();
    }
    m1 = wave_sum(m1);
    m2 = wave_sum(m2);
    if ((threadIdx.x & 63u) == 0u) { total[0][threadIdx.x >> 6] = m1; total[1][threadIdx.x >> 6] = m2; }
    __syncthreads();
    if (threadIdx.x >= 2u) return;
    const float inv = 1.0f / ((float)A.P * (float)A.w);
    A.group_sums[(uint64_t)blockIdx.x * 2u + threadIdx.x] = (total[threadIdx.x][0] + total[threadIdx.x][1] + total[threadIdx.x][2] + total[threadIdx.x][3]) * inv;
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
// Held: whole groups of 64 channels and more a workgroup, so that a row of it is a cache line, of at most `most` rows a team.
struct GroupNormPlan {
    bool held;
    uint32_t lanes, threads, rows_of_team, groups, slabs;    // held
    uint32_t blocks, chunks, rows;                           // else
};
static GroupNormPlan group_norm_plan(uint32_t B, uint32_t P, uint32_t C, uint32_t G, uint32_t most) {
    GroupNormPlan L = {};
    const uint32_t w = C / G;
    L.groups = std::min(G, std::max(1u, (64u + w - 1u) / w));
    L.slabs = (G + L.groups - 1u) / L.groups;
    const uint32_t width = L.groups * w;
    if (width <= kMostSlab) {
        L.lanes = power_of_two((width + 7u) / 8u);
        L.threads = 256u;
        while (L.threads < kMostThreads && (uint64_t)P > (uint64_t)(L.threads / L.lanes) * std::min(most, 4u)) L.threads *= 2u;
        const uint64_t teams = L.threads / L.lanes;
        L.held = P <= teams * most;
        L.rows_of_team = (uint32_t)((P + teams - 1u) / teams);
    }
    if (L.held) return L;
    const uint32_t pieces = (C + 7u) / 8u;
    L.lanes = power_of_two(std::min(pieces, 32u));
    L.threads = 256u;
    L.blocks = (pieces + L.lanes - 1u) / L.lanes;
    const uint32_t teams = 256u / L.lanes;
    // eight workgroups a compute unit, of at least eight rows a team
    const uint64_t want = std::max<uint64_t>(1, 2048u / std::max<uint64_t>(1, (uint64_t)B * L.blocks));
    L.chunks = (uint32_t)std::min<uint64_t>(want, (P + teams * 8u - 1u) / (teams * 8u));
    L.rows = (P + L.chunks - 1u) / L.chunks;
    L.chunks = (P + L.rows - 1u) / L.rows;
    return L;
}
static uint32_t most_rows(int dtype, bool backward) { return (dtype == VGC_F32 ? 8u : 16u) / (backward ? 2u : 1u); }

struct GroupNormSpace { size_t chunk_sums, sums, group_sums, total; };
static GroupNormSpace group_norm_space(const GroupNormPlan& L, uint32_t B, uint32_t C, uint32_t G, bool backward) {
    GroupNormSpace S;
    size_t off = 0;
    S.chunk_sums = off; if (!L.held) off = align_up(off + (size_t)B * L.chunks * 2u * C * sizeof(float), 256);
    S.sums = off; if (backward) off = align_up(off + (size_t)B * 2u * C * sizeof(float), 256);
    S.group_sums = off; if (backward && !L.held) off += (size_t)B * 2u * G * sizeof(float);
    S.total = off;
    return S;
}
size_t group_norm_workspace_bytes(int dtype, uint32_t B, uint32_t P, uint32_t C, uint32_t G) {
    return group_norm_space(group_norm_plan(B, P, C, G, most_rows(dtype, false)), B, C, G, false).total;
}
size_t group_norm_backward_workspace_bytes(int dtype, uint32_t B, uint32_t P, uint32_t C, uint32_t G) {
    return group_norm_space(group_norm_plan(B, P, C, G, most_rows(dtype, true)), B, C, G, true).total;
}

// Calls launch(args, samples) for ranges of samples, of `each` workgroups a sample at most, that a launch can hold.
template <typename Launch>
static int by_samples(const GroupNormArgs& all, size_t size, uint64_t each, const GroupNormPlan& L, Launch launch) {
    const uint32_t most = (uint32_t)std::max<uint64_t>(1, (1u << 22) / each);
    for (uint32_t b = 0; b < all.B; b += std::min(most, all.B - b)) {
        GroupNormArgs A = all;
        const size_t at = (size_t)b * A.P * A.C * size;
        A.B = std::min(most, all.B - b);
        A.x = (const char*)all.x + at;
        if (all.dy) A.dy = (const char*)all.dy + at;
        A.out = (char*)all.out + at;
        const size_t group = (size_t)b * A.G;
        if (all.mean) { A.mean += group; A.rstd += group; }
        if (all.mean_out) { A.mean_out += group; A.rstd_out += group; }
        if (!L.held) A.chunk_sums += (size_t)b * L.chunks * 2u * A.C;
        if (all.sums) A.sums += (size_t)b * 2u * A.C;
        if (all.group_sums) A.group_sums += group * 2u;
        const int rc = launch(A, A.B);
        if (rc != VGC_OK) return rc;
    }
    return VGC_OK;
}

static void place(GroupNormArgs& A, const GroupNormPlan& L) {
    A.lanes = L.lanes; A.blocks = L.blocks; A.chunks = L.chunks; A.rows = L.rows; A.groups = L.groups; A.slabs = L.slabs;
}

template <typename T>
static int launch_group_norm_of(GroupNormArgs& all, const GroupNormPlan& L, hipStream_t stream) {
    if (L.held)
        return by_samples(all, sizeof(T), L.slabs, L, [&](const GroupNormArgs& A, uint32_t B) {
#define VGC_LAUNCH(NV) hipLaunchKernelGGL((k_group_norm<T, NV>), dim3(B * L.slabs), dim3(L.threads), 0, stream, A)
            if (L.rows_of_team <= 2u) VGC_LAUNCH(2);
            else if (L.rows_of_team <= 4u) VGC_LAUNCH(4);
            else if (L.rows_of_team <= 8u) VGC_LAUNCH(8);
            else if constexpr (sizeof(T) == 2) VGC_LAUNCH(16);
#undef VGC_LAUNCH
            return hip_check(hipGetLastError(), "launch k_group_norm");
        });
    return by_samples(all, sizeof(T), std::max(L.blocks * L.chunks, all.G), L, [&](GroupNormArgs A, uint32_t B) {
        const dim3 grid(B * L.blocks * L.chunks);
        hipLaunchKernelGGL(k_group_norm_moments<T>, grid, dim3(256), 0, stream, A);
        int rc = hip_check(hipGetLastError(), "launch k_group_norm_moments");
        if (rc != VGC_OK) return rc;
        hipLaunchKernelGGL(k_group_norm_join, dim3(B * A.G), dim3((uint64_t)L.chunks * A.w > 256u ? 256 : 64), 0, stream, A);
        if ((rc = hip_check(hipGetLastError(), "launch k_group_norm_join")) != VGC_OK) return rc;
        A.mean = A.mean_out;
        A.rstd = A.rstd_out;
        hipLaunchKernelGGL(k_group_norm_apply<T>, grid, dim3(256), 0, stream, A);
        return hip_check(hipGetLastError(), "launch k_group_norm_apply");
    });
}

int launch_group_norm(int dtype, const void* x, uint32_t B, uint32_t P, uint32_t C, uint32_t G, const float* gamma, const float* beta, float eps, int act,
                      void* y, float* mean, float* rstd, void* workspace, hipStream_t stream) {
    const GroupNormPlan L = group_norm_plan(B, P, C, G, most_rows(dtype, false));
    GroupNormArgs A = {};
    A.x = x; A.gamma = gamma; A.beta = beta; A.mean_out = mean; A.rstd_out = rstd; A.out = y;
    A.chunk_sums = static_cast<float*>(workspace);
    A.B = B; A.P = P; A.C = C; A.G = G; A.w = C / G; A.act = (uint32_t)act; A.eps = eps;
    place(A, L);
    return dtype == VGC_F32 ? launch_group_norm_of<float>(A, L, stream) : launch_group_norm_of<uint16_t>(A, L, stream);
}

template <typename T>
static int launch_group_norm_backward_of(GroupNormArgs& all, const GroupNormPlan& L, hipStream_t stream) {
    if (L.held)
        return by_samples(all, sizeof(T), L.slabs, L, [&](const GroupNormArgs& A, uint32_t B) {
#define VGC_LAUNCH(NV) hipLaunchKernelGGL((k_group_norm_backward<T, NV>), dim3(B * L.slabs), dim3(L.threads), 0, stream, A)
            if (L.rows_of_team <= 2u) VGC_LAUNCH(2);
            else if (L.rows_of_team <= 4u) VGC_LAUNCH(4);
            else if constexpr (sizeof(T) == 2) VGC_LAUNCH(8);
#undef VGC_LAUNCH
            return hip_check(hipGetLastError(), "launch k_group_norm_backward");
        });
    return by_samples(all, sizeof(T), std::max(L.blocks * L.chunks, all.G), L, [&](const GroupNormArgs& A, uint32_t B) {
        const dim3 grid(B * L.blocks * L.chunks);
        hipLaunchKernelGGL((k_group_norm_backward_rows<T, true>), grid, dim3(256), 0, stream, A);
        int rc = hip_check(hipGetLastError(), "launch k_group_norm_backward_rows");
        if (rc != VGC_OK) return rc;
        hipLaunchKernelGGL(k_group_norm_backward_join, dim3(B * A.G), dim3(256), 0, stream, A);
        if ((rc = hip_check(hipGetLastError(), "launch k_group_norm_backward_join")) != VGC_OK) return rc;
        hipLaunchKernelGGL((k_group_norm_backward_rows<T, false>), grid, dim3(256), 0, stream, A);
        return hip_check(hipGetLastError(), "launch k_group_norm_backward_rows");
    });
}

int launch_group_norm_backward(int dtype, const void* dy, const void* x, const float* mean, const float* rstd, const float* gamma, const float* beta,
                               int act, uint32_t B, uint32_t P, uint32_t C, uint32_t G, float c, void* dx, float* g_gamma, float* s_gamma, float* g_beta,
                               float* s_beta, void* workspace, hipStream_t stream) {
    const GroupNormPlan L = group_norm_plan(B, P, C, G, most_rows(dtype, true));
    const GroupNormSpace S = group_norm_space(L, B, C, G, true);
    char* ws = static_cast<char*>(workspace);
    GroupNormArgs A = {};
    A.x = x; A.dy = dy; A.gamma = gamma; A.beta = beta; A.mean = mean; A.rstd = rstd; A.out = dx;
    A.chunk_sums = (float*)(ws + S.chunk_sums);
    A.sums = (float*)(ws + S.sums);
    if (!L.held) A.group_sums = (float*)(ws + S.group_sums);
    A.B = B; A.P = P; A.C = C; A.G = G; A.w = C / G; A.act = (uint32_t)act;
    place(A, L);
    const int rc = dtype == VGC_F32 ? launch_group_norm_backward_of<float>(A, L, stream) : launch_group_norm_backward_of<uint16_t>(A, L, stream);
    if (rc != VGC_OK) return rc;
    return launch_column_sums(A.sums, 2, 0, B, 1, C, false, c, g_gamma, s_gamma, g_beta, s_beta, stream);
}

}  // namespace vgc
