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
    bool past;                // the result is stored past the caches
};

// gamma xhat + beta, rounded after each operation in both passes: relu's slope is decided by the sign that the forward pass saw, which with one
// rounding less would be another once in some 10^8 elements.
__device__ __forceinline__ float scaled(float xhat, float gamma, float beta) { return xhat * gamma + beta; }

__device__ __forceinline__ uint32_t at_most(uint32_t a, uint32_t b) { return a < b ? a : b; }

// Sums of two vectors of channels (or of one: b NULL) over whole groups of w, a wave a group: into ga and gb.  Ends with a barrier.
template <bool kTwo, typename Weight>
__device__ __forceinline__ void sums_of_groups(const float* a, const float* b, uint32_t w, uint32_t groups, float* ga, float* gb, Weight weight) {
    const uint32_t lane = threadIdx.x & 63u, waves = blockDim.x / 64u;
    for (uint32_t q = threadIdx.x >> 6; q < groups; q += waves) {
        float s = 0.f, t = 0.f;
        for (uint32_t c = lane; c < w; c += 64u) {
            const float of = weight(q * w + c);
            s = __builtin_fmaf(of, a[q * w + c], s);
            if (kTwo) t = __builtin_fmaf(of, b[q * w + c], t);
        }
        s = wave_sum(s);
        if (kTwo) t = wave_sum(t);
        if (lane == 0) { ga[q] = s; if (kTwo) gb[q] = t; }
    }
    __syncthreads();
}

// ---- a sample's whole groups in one workgroup ---------------------------------------------------------------------------------
// kNV rows of a team are held as they are in memory.  A workgroup's reading, sums and writing follow each other, with one or two workgroups a
// compute unit, which bounds them (32 x 49 x 2048 float32 in 32 groups 8.5 us, 64 x 784 x 512 bfloat16 a call of 32-34, both 3.0-3.2 TB/s of the 5.1 that a
// copy reaches; as chunks 16.3 and 39.5.  Backward 32 x 196 x 1024 float32 27.5, as chunks 37).
// How a workgroup's groups lie in its lanes decides how a group's sum is formed: by channels, which may belong to any group; a lane's eight
// channels of one group, then by lanes; or all lanes' of one.
enum { kByChannel, kByLane, kOneGroup };
constexpr uint32_t kMostThreads = 1024, kMostSlab = 512;     // threads, channels

// The sum over the group that a lane's channels belong to, for each of them; `out` (by group) keeps it until the next but one barrier.
template <int kMode> struct GroupSums {
    float *sh, *part, *chan, *grp;
    uint32_t lanes, w, groups;
    __device__ __forceinline__ void of(const float (&v)[8]) const {
        if constexpr (kMode == kByChannel) {
            const float one[1][8] = {{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}};
            channel_sums<1>(one, lanes, sh, part, chan);
            sums_of_groups<false>(chan, nullptr, w, groups, grp, nullptr, [](uint32_t) { return 1.f; });
            return;
        }
        const float sum = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, waves = blockDim.x / 64u;
        if constexpr (kMode == kOneGroup) {
            const float all = wave_sum(sum);
            if (lane == 0) part[wave] = all;
            __syncthreads();
            float total = 0.f;
            for (uint32_t i = 0; i < waves; ++i) total += part[i];
            __syncthreads();
            if (threadIdx.x == 0) grp[0] = total;
            __syncthreads();
        } else {
            part[threadIdx.x] = sum;
            __syncthreads();
            const uint32_t each = w / 8u, entries = blockDim.x / lanes * each;         // lanes of a group in a team, in all
            for (uint32_t q = wave; q < groups; q += waves) {
                float s = 0.f;
                for (uint32_t e = lane; e < entries; e += 64u) s += part[e / each * lanes + q * each + e % each];
                s = wave_sum(s);
                if (lane == 0) grp[q] = s;
            }
            __syncthreads();
        }
    }
};

template <typename T, int kNV, int kMode, int kThreads>
__global__ __launch_bounds__(kThreads) void k_group_norm(GroupNormArgs A) {
    __shared__ float sh[kMode == kByChannel ? kThreads * 8 : 1], part[kThreads], chan[kMode == kByChannel ? kMostSlab : 1], grp[64];
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
    uint32_t of[kMode == kByChannel ? 8 : 1];                // group of a channel
#pragma unroll
    for (int k = 0; k < (kMode == kByChannel ? 8 : 1); ++k) of[k] = k < n && kMode != kOneGroup ? (own + k) / A.w : 0u;
    float ga[8], be[8];
    widen8(load8(A.gamma + c0 + own, n), ga);
    widen8(load8(A.beta + c0 + own, n), be);
    const float inv = 1.0f / ((float)A.P * (float)A.w);
    const GroupSums<kMode> sums = {sh, part, chan, grp, A.lanes, A.w, groups};
    float f[8], v[8] = {};
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        clip8(raw[i], n);
        widen8(raw[i], f);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += f[k];
    }
    sums.of(v);
    constexpr int kM = kMode == kByChannel ? 8 : 1;
    float mean[kM], rstd[kM];
#pragma unroll
    for (int k = 0; k < kM; ++k) mean[k] = grp[of[k]] * inv;
    const float own_mean = threadIdx.x < groups ? grp[threadIdx.x] * inv : 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.f;
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        widen8(raw[i], f);
        if (team + i * teams < A.P)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float d = k < n ? f[k] - mean[kM == 8 ? k : 0] : 0.f;
                v[k] = __builtin_fmaf(d, d, v[k]);
            }
    }
    sums.of(v);
#pragma unroll
    for (int k = 0; k < kM; ++k) rstd[k] = 1.0f / sqrtf(grp[of[k]] * inv + A.eps);
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
        for (int k = 0; k < 8; ++k) f[k] = scaled((f[k] - mean[kM == 8 ? k : 0]) * rstd[kM == 8 ? k : 0], ga[k], be[k]);
        apply_act((int)A.act, f);
        store8(y + (uint64_t)p * A.C, f, n);
    }
}

// The groups' mean and rstd (kM = 1: one group's), gamma and beta for a lane's channels c0 .. (n of them).
template <int kM> struct Channels {
    float mean[kM], rstd[kM], gamma[8], beta[8];
    __device__ __forceinline__ Channels(const GroupNormArgs& A, uint32_t b, uint32_t c0, int n) {
        widen8(load8(A.gamma + c0, n), gamma);
        widen8(load8(A.beta + c0, n), beta);
#pragma unroll
        for (int k = 0; k < kM; ++k) {
            mean[k] = rstd[k] = 0.f;
            if (k >= n) continue;
            const uint64_t at = (uint64_t)b * A.G + (c0 + k) / A.w;
            mean[k] = A.mean[at];
            rstd[k] = A.rstd[at];
        }
    }
    __device__ __forceinline__ float xhat(float x, int k) const { return (x - mean[kM == 8 ? k : 0]) * rstd[kM == 8 ? k : 0]; }
};
// x becomes xhat, d becomes e = dy act'(gamma xhat + beta).
template <int kM>
__device__ __forceinline__ void through_act(const GroupNormArgs& A, const Channels<kM>& K, float (&x)[8], float (&d)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = K.xhat(x[k], k);
    if (A.act == VGC_ACT_NONE) return;
    float t[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) t[k] = scaled(x[k], K.gamma[k], K.beta[k]);
    apply_slope((int)A.act, t, d);
}

template <typename T, int kNV, int kThreads, int kM>
__global__ __launch_bounds__(kThreads) void k_group_norm_backward(GroupNormArgs A) {
    __shared__ float sh[2 * kThreads * 8], part[2 * kThreads], chan[2][kMostSlab], grp[2][64];
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
    const Channels<kM> K(A, b, c0 + own, n);
    float x[8], d[8], v[2][8] = {};
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        if (team + i * teams >= A.P) continue;
        clip8(rd[i], n);
        clip8(rx[i], n);
        widen8(rx[i], x);
        widen8(rd[i], d);
        through_act(A, K, x, d);
#pragma unroll
        for (int k = 0; k < 8; ++k) { v[0][k] = __builtin_fmaf(d[k], x[k], v[0][k]); v[1][k] += d[k]; }
    }
    channel_sums<2>(v, A.lanes, sh, part, chan[0], chan[1]);
    const float* gamma = A.gamma + c0;
    sums_of_groups<true>(chan[1], chan[0], A.w, groups, grp[0], grp[1], [&](uint32_t c) { return gamma[c]; });
    for (uint32_t c = threadIdx.x; c < 2u * width; c += blockDim.x) {
        const uint32_t v = c >= width, ch = c - v * width;
        A.sums[((uint64_t)b * 2u + v) * A.C + c0 + ch] = chan[v][ch];
    }
    if (n <= 0) return;
    const float inv = 1.0f / ((float)A.P * (float)A.w);
    float m1[kM], m2[kM];
#pragma unroll
    for (int k = 0; k < kM; ++k) {
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
        for (int k = 0; k < 8; ++k) {
            const int g = kM == 8 ? k : 0;
            d[k] = K.rstd[g] * __builtin_fmaf(-x[k], m2[g], __builtin_fmaf(d[k], K.gamma[k], -m1[g]));
        }
        store8(static_cast<T*>(A.out) + at + (uint64_t)p * A.C, d, n);
    }
}

// ---- samples beyond that: sums by channel and chunk, then the result ------------------------------------------------------------
// Workgroup (sample, block of columns, chunk of positions): teams take the chunk's rows in turn, two sets of kRows of them in turn in flight.
// Both passes are bound by memory (64 x 50176 x 64 bfloat16 with relu, 411 MB: 211 us in two halves of the samples, of each the moments 40, 5.1 TB/s, and the result
// 65, 6.3 TB/s, from the last-level cache for what it keeps.  Backward, 32 x 3136 x 256 float32 with silu, 103 MB an array: 97 us).
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
template <typename T> struct Stream { static constexpr int kRows = sizeof(T) == 2 ? 4 : 2; };
template <typename T, bool kWhole, int kRows, int kArrays>
__device__ __forceinline__ RowStream<T, kWhole, kRows, kArrays> rows_of(const GroupNormArgs& A, const Place& L, const void* a, const void* b) {
    const uint64_t row0 = (uint64_t)L.b * A.P;
    return RowStream<T, kWhole, kRows, kArrays>(static_cast<const T*>(a) + row0 * A.C, static_cast<const T*>(b) + (b ? row0 * A.C : 0u), A.C, L.c0, L.p0 + L.team, L.p1, L.teams,
                                                (uint64_t)A.B * A.P - row0);
}

// Mean and sum of squares about it, by channel.  A lane's sums are relative to the mean of its first rows (kRows of them): what the sum of
// squares then loses to the difference of that mean and its whole mean is at most the share of those rows, whatever the values.  Lanes are joined as
// (count, mean, squares), so that a large mean costs no digits.
template <typename T, bool kWhole>
__global__ __launch_bounds__(256) void k_group_norm_moments(GroupNormArgs A) {
    constexpr int kRows = Stream<T>::kRows;
    __shared__ float sm[2048], sq[2048], pm[256], pq[256];
    const Place L = place_of(A);
    auto X = rows_of<T, kWhole, kRows, 1>(A, L, A.x, nullptr);
    float base[8] = {}, s1[8] = {}, s2[8] = {}, f[8];
    const uint32_t count = rows_of_team(L.p1 - L.p0, L.team, L.teams);
    const uint32_t first = at_most(count, kRows);
    X.begin();
    if (first != 0u) {
        const float inv = 1.0f / (float)first;
#pragma unroll
        for (uint32_t i = 0; i < kRows; ++i) {
            if (i >= first) continue;
            widen8(kWhole ? X.set[0][0][i] : X.at(0, X.p + i * X.step), f);
#pragma unroll
            for (int k = 0; k < 8; ++k) base[k] += f[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) base[k] *= inv;
    }
    X.each([&](uint32_t, const Raw8<T> (&x)[1]) {
        float f[8];
        widen8(x[0], f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float d = f[k] - base[k];
            s1[k] += d;
            s2[k] = __builtin_fmaf(d, d, s2[k]);
        }
    });
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
    const uint32_t each = rows_here / L.teams, more = rows_here - each * L.teams;             // rows of a team; teams with one more
    float total = 0.f, mean = 0.f, squares = 0.f;
    for (uint32_t t = 0; t < 8u; ++t) {
        const float m = (float)(each + (sub * 8u + t < more ? 1u : 0u));
        total += m;
        mean = __builtin_fmaf(m, sm[(sub * 8u + t) * S + c], mean);
    }
    if (total > 0.f) mean /= total;
    for (uint32_t t = 0; t < 8u; ++t) {
        const float m = (float)(each + (sub * 8u + t < more ? 1u : 0u)), d = sm[(sub * 8u + t) * S + c] - mean;
        if (m > 0.f) squares += __builtin_fmaf(m * d, d, sq[(sub * 8u + t) * S + c]);
    }
    if (subs > 1u) {
        pm[threadIdx.x] = mean;
        pq[threadIdx.x] = squares;
        __syncthreads();
        if (threadIdx.x >= S) return;
        auto rows_of_sub = [&](uint32_t q) { return (float)(each * 8u + (more > q * 8u ? min(more - q * 8u, 8u) : 0u)); };
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

// A group's moments from those of its channels and chunks; in 64 bits, so that mean^2 may be subtracted.  (With 64 threads for any number of
// entries 2 x 47061 x 296 float32 waited 150 us for its two groups of many chunks.)
__global__ __launch_bounds__(1024) void k_group_norm_join(GroupNormArgs A) {
    __shared__ double sh[2][16];
    const uint32_t b = blockIdx.x / A.G, q = blockIdx.x - b * A.G, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const float* in = A.chunk_sums + (uint64_t)b * A.chunks * 2u * A.C + q * A.w;
    double s1 = 0., s2 = 0.;
#pragma unroll 4
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

template <typename T, bool kWhole, int kM>
__global__ __launch_bounds__(256) void k_group_norm_apply(GroupNormArgs A) {
    const Place L = place_of(A);
    if (!kWhole && L.n <= 0) return;
    auto X = rows_of<T, kWhole, Stream<T>::kRows, 1>(A, L, A.x, nullptr);
    T* y = static_cast<T*>(A.out) + (uint64_t)L.b * A.P * A.C + L.c0;
    X.begin();
    const Channels<kM> K(A, L.b, L.c0, L.n);
    X.each([&](uint32_t p, const Raw8<T> (&x)[1]) {
        float f[8];
        widen8(x[0], f);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = scaled(K.xhat(f[k], k), K.gamma[k], K.beta[k]);
        apply_act((int)A.act, f);
        if (L.n > 0) store8_to(y + (uint64_t)p * A.C, f, L.n, A.past);
    });
}

// kSums: G_z and H_z of the chunk; else dx.  (32 x 3136 x 256 float32: the sums 39 us, 5.2 TB/s, dx 49.)
template <typename T, bool kWhole, int kM, bool kSums>
__global__ __launch_bounds__(256) void k_group_norm_backward_rows(GroupNormArgs A) {
    __shared__ float sh[kSums ? 4096 : 1], part[kSums ? 512 : 1], chan[2][kSums ? 256 : 1];
    const Place L = place_of(A);
    if (!kSums && !kWhole && L.n <= 0) return;
    auto X = rows_of<T, kWhole, Stream<T>::kRows / 2, 2>(A, L, A.x, A.dy);
    X.begin();
    const Channels<kM> K(A, L.b, L.c0, L.n);
    float m1[kM] = {}, m2[kM] = {};
    if (!kSums)
#pragma unroll
        for (int k = 0; k < kM; ++k)
            if (k < L.n) {
                const float* g = A.group_sums + ((uint64_t)L.b * A.G + (L.c0 + k) / A.w) * 2u;
                m1[k] = g[0];
                m2[k] = g[1];
            }
    float v[2][8] = {};
    T* out = static_cast<T*>(A.out) + (uint64_t)L.b * A.P * A.C + L.c0;
    X.each([&](uint32_t p, const Raw8<T> (&in)[2]) {
        float x[8], d[8];
        widen8(in[0], x);
        widen8(in[1], d);
        through_act(A, K, x, d);
        if (kSums) {
#pragma unroll
            for (int k = 0; k < 8; ++k) { v[0][k] = __builtin_fmaf(d[k], x[k], v[0][k]); v[1][k] += d[k]; }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int g = kM == 8 ? k : 0;
                d[k] = K.rstd[g] * __builtin_fmaf(-x[k], m2[g], __builtin_fmaf(d[k], K.gamma[k], -m1[g]));
            }
            if (L.n > 0) store8_to(out + (uint64_t)p * A.C, d, L.n, A.past);
        }
    });
    if (!kSums) return;
    const uint32_t first = L.c0 - (threadIdx.x % A.lanes) * 8u, c = first + threadIdx.x;
    float* sums = A.chunk_sums + ((uint64_t)L.b * A.chunks + L.chunk) * 2u * A.C;
    channel_sums<2>(v, A.lanes, sh, part, chan[0], chan[1]);
    if (threadIdx.x >= A.lanes * 8u || c >= A.C) return;
    sums[c] = chan[0][threadIdx.x];
    sums[A.C + c] = chan[1][threadIdx.x];
}

// G_z and H_z of a group's channels from their chunks, and the group's two sums.  Threads: up to 64 channels, the others share their chunks; a thread adds every
// `subs`th in turn, then the channel's first its fellows' sums.
__global__ __launch_bounds__(1024) void k_group_norm_backward_join(GroupNormArgs A) {
    __shared__ float sh[2][1024], total[2][16];
    const uint32_t b = blockIdx.x / A.G, q = blockIdx.x - b * A.G, threads = blockDim.x;
    uint32_t wp = 1;
    while (wp < A.w && wp < 64u) wp *= 2u;
    const uint32_t ch = threadIdx.x % wp, sub = threadIdx.x / wp, subs = threads / wp;
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
        for (uint32_t n = subs; n > 1u;) {                   // (subs: a power of two)
            const uint32_t half = n / 2u;
            if (sub < half) {
                sh[0][threadIdx.x] += sh[0][threadIdx.x + half * wp];
                sh[1][threadIdx.x] += sh[1][threadIdx.x + half * wp];
            }
            __syncthreads();
            n = half;
        }
        if (sub == 0u && c < A.w) {
            g = sh[0][threadIdx.x];
            h = sh[1][threadIdx.x];
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
    float sum = 0.f;
    for (uint32_t v = 0; v < threads / 64u; ++v) sum += total[threadIdx.x][v];
    A.group_sums[(uint64_t)blockIdx.x * 2u + threadIdx.x] = sum * (1.0f / ((float)A.P * (float)A.w));
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
// Held: whole groups of a cache line's channels and more a workgroup (us; float32, 32 x 784 x 512 in 32 groups, lines of 32 channels 32.2, 64 39.1;
// bfloat16, 64 x 784 x 512, of 64 34.3, 32 46), with as many threads as leave a team few rows.  most: rows that a team can hold, with 512 threads
// and fewer and with 1024, whose lanes have 128 registers: backward half as many, and by channel, which takes more of them, none.  (Forward, 1024 threads hold whatever
// 512 would.)
// Else: workgroups to fill the compute units, and as many samples at a time as the last-level cache keeps of them between the two passes, that is
// somewhat less than its 256 MB (us, 64 x 50176 x 64 bfloat16: 210 MB in 2048 workgroups 219, in 1024 232; 128 MB 255; all at once 246).
struct GroupNormPlan {
    bool held;
    uint32_t lanes, threads, rows_of_team, groups, slabs;    // held
    uint32_t blocks, chunks, rows;                           // else
    uint32_t samples;                                        // at a time
};
constexpr uint32_t kGroups = 2048;
constexpr uint64_t kSlice = 210ull << 20;
static GroupNormPlan group_norm_plan(int dtype, bool backward, uint32_t B, uint32_t P, uint32_t C, uint32_t G) {
    GroupNormPlan L = {};
    const uint32_t w = C / G, line = dtype == VGC_F32 ? 32u : 64u;
    L.groups = std::min(G, std::max(1u, (line + w - 1u) / w));
    L.slabs = (G + L.groups - 1u) / L.groups;
    const uint32_t width = L.groups * w, wide = dtype == VGC_F32 ? 2u : 1u;
    const uint32_t most = 8u / wide, most_1024 = backward ? (w % 8u == 0u ? 4u / wide : 0u) : most, few = backward ? 4u / wide : 4u;
    if (width <= kMostSlab) {
        L.lanes = power_of_two((width + 7u) / 8u);
        for (L.threads = 256u; L.threads < kMostThreads && P > (uint64_t)(L.threads / L.lanes) * few;) L.threads *= 2u;
        if (backward && L.threads == kMostThreads && P > (uint64_t)(L.threads / L.lanes) * most_1024) L.threads = 512u;
        const uint32_t teams = L.threads / L.lanes;
        L.rows_of_team = (P + teams - 1u) / teams;
        L.held = L.rows_of_team <= (L.threads == kMostThreads ? most_1024 : most);
    }
    if (L.held) { L.samples = std::min(B, std::max(1u, (1u << 20) / L.slabs)); return L; }      // (a launch has fewer than 2^32 threads)
    const uint32_t pieces = (C + 7u) / 8u;
    L.lanes = power_of_two(std::min(pieces, 32u));
    L.threads = 256u;
    L.blocks = (pieces + L.lanes - 1u) / L.lanes;
    const uint32_t teams = 256u / L.lanes;
    const uint64_t sample = (uint64_t)P * C * (dtype == VGC_F32 ? 4u : 2u) * (backward ? 2u : 1u), most_samples = std::max<uint64_t>(1, kSlice / sample);
    const uint32_t times = (uint32_t)((B + most_samples - 1u) / most_samples);
    L.samples = std::min((B + times - 1u) / times, std::max(1u, (1u << 20) / std::max(L.blocks, G)));
    const uint64_t want = std::max<uint64_t>(1, kGroups / std::max<uint64_t>(1, (uint64_t)L.samples * L.blocks));
    L.chunks = (uint32_t)std::min<uint64_t>(std::min<uint64_t>(want, 256u), (P + teams * 2u - 1u) / (teams * 2u));      // (256: of which a group's join has to read all)
    const uint32_t batch = teams * (dtype == VGC_F32 ? 2u : 4u) * (backward ? 1u : 2u);      // (whole batches but for the sample's last)
    L.rows = (P - 1u) / L.chunks + 1u;
    if (L.rows > 2u * batch) L.rows = (L.rows + batch / 2u) / batch * batch;
    if ((P - 1u) / L.rows >= 256u) L.rows += batch;         // (rounded down)
    L.chunks = (P - 1u) / L.rows + 1u;
    return L;
}

void group_norm_form(int dtype, bool backward, uint32_t B, uint32_t P, uint32_t C, uint32_t G, uint32_t* form) {
    const GroupNormPlan L = group_norm_plan(dtype, backward, B, P, C, G);
    form[0] = L.held; form[1] = L.threads; form[2] = L.rows_of_team; form[3] = L.groups; form[4] = L.samples; form[5] = L.chunks;
}

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
    return group_norm_space(group_norm_plan(dtype, false, B, P, C, G), B, C, G, false).total;
}
size_t group_norm_backward_workspace_bytes(int dtype, uint32_t B, uint32_t P, uint32_t C, uint32_t G) {
    return group_norm_space(group_norm_plan(dtype, true, B, P, C, G), B, C, G, true).total;
}

// Calls launch(args, samples) for the plan's samples at a time.
template <typename Launch>
static int by_samples(const GroupNormArgs& all, size_t size, const GroupNormPlan& L, Launch launch) {
    const uint64_t sample = (uint64_t)all.P * all.C * size;
    for (uint32_t b = 0; b < all.B; b += std::min(L.samples, all.B - b)) {
        GroupNormArgs A = all;
        const size_t at = (size_t)b * sample;
        A.B = std::min(L.samples, all.B - b);
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

// Threads that join a group's chunks: four entries each.
static uint32_t join_threads(const GroupNormPlan& L, uint32_t w) {
    const uint64_t entries = (uint64_t)L.chunks * w;
    return entries <= 256u ? 64u : entries <= 1024u ? 256u : 1024u;
}
// Whether a lane's eight channels belong to one group wherever its piece lies.
static bool by_lane(const GroupNormArgs& A) { return A.w % 8u == 0u; }

template <typename T>
static int launch_group_norm_of(const GroupNormArgs& all, const GroupNormPlan& L, hipStream_t stream) {
    if (L.held)
        return by_samples(all, sizeof(T), L, [&](const GroupNormArgs& A, uint32_t B) {
#define VGC_LAUNCH(NV, THREADS) do { \
            if (L.groups == 1u) hipLaunchKernelGGL((k_group_norm<T, NV, kOneGroup, THREADS>), dim3(B * L.slabs), dim3(L.threads), 0, stream, A); \
            else if (by_lane(A)) hipLaunchKernelGGL((k_group_norm<T, NV, kByLane, THREADS>), dim3(B * L.slabs), dim3(L.threads), 0, stream, A); \
            else hipLaunchKernelGGL((k_group_norm<T, NV, kByChannel, THREADS>), dim3(B * L.slabs), dim3(L.threads), 0, stream, A); } while (0)
            if (L.rows_of_team <= 2u) VGC_LAUNCH(2, 1024);
            else if (sizeof(T) == 4 || L.rows_of_team <= 4u) VGC_LAUNCH(4, 1024);
            else if constexpr (sizeof(T) == 2) VGC_LAUNCH(8, 1024);
#undef VGC_LAUNCH
            return hip_check(hipGetLastError(), "launch k_group_norm");
        });
    return by_samples(all, sizeof(T), L, [&](GroupNormArgs A, uint32_t B) {
        const dim3 grid(B * L.blocks * L.chunks);
        const bool whole = A.C % 8u == 0u;
        if (whole) hipLaunchKernelGGL((k_group_norm_moments<T, true>), grid, dim3(256), 0, stream, A);
        else hipLaunchKernelGGL((k_group_norm_moments<T, false>), grid, dim3(256), 0, stream, A);
        int rc = hip_check(hipGetLastError(), "launch k_group_norm_moments");
        if (rc != VGC_OK) return rc;
        hipLaunchKernelGGL(k_group_norm_join, dim3(B * A.G), dim3(join_threads(L, A.w)), 0, stream, A);
        if ((rc = hip_check(hipGetLastError(), "launch k_group_norm_join")) != VGC_OK) return rc;
        A.mean = A.mean_out;
        A.rstd = A.rstd_out;
        if (by_lane(A)) hipLaunchKernelGGL((k_group_norm_apply<T, true, 1>), grid, dim3(256), 0, stream, A);
        else if (whole) hipLaunchKernelGGL((k_group_norm_apply<T, true, 8>), grid, dim3(256), 0, stream, A);
        else hipLaunchKernelGGL((k_group_norm_apply<T, false, 8>), grid, dim3(256), 0, stream, A);
        return hip_check(hipGetLastError(), "launch k_group_norm_apply");
    });
}

int launch_group_norm(int dtype, const void* x, uint32_t B, uint32_t P, uint32_t C, uint32_t G, const float* gamma, const float* beta, float eps, int act,
                      void* y, float* mean, float* rstd, void* workspace, hipStream_t stream) {
    const GroupNormPlan L = group_norm_plan(dtype, false, B, P, C, G);
    GroupNormArgs A = {};
    A.x = x; A.gamma = gamma; A.beta = beta; A.mean_out = mean; A.rstd_out = rstd; A.out = y;
    A.chunk_sums = static_cast<float*>(workspace);
    A.B = B; A.P = P; A.C = C; A.G = G; A.w = C / G; A.act = (uint32_t)act; A.eps = eps;
    place(A, L);
    A.past = past_caches(y, C, (uint64_t)B * P * C * (dtype == VGC_F32 ? 4u : 2u) * 2u);
    return dtype == VGC_F32 ? launch_group_norm_of<float>(A, L, stream) : launch_group_norm_of<uint16_t>(A, L, stream);
}

template <typename T>
static int launch_group_norm_backward_of(const GroupNormArgs& all, const GroupNormPlan& L, hipStream_t stream) {
    if (L.held)
        return by_samples(all, sizeof(T), L, [&](const GroupNormArgs& A, uint32_t B) {
            constexpr int kFew = sizeof(T) == 2 ? 4 : 2;
#define VGC_LAUNCH(NV, THREADS, M) hipLaunchKernelGGL((k_group_norm_backward<T, NV, THREADS, M>), dim3(B * L.slabs), dim3(L.threads), 0, stream, A)
#define VGC_ROWS(M) do { if (L.rows_of_team <= kFew / 2) VGC_LAUNCH(kFew / 2, 512, M); else VGC_LAUNCH(kFew, 512, M); } while (0)
            if (L.threads == kMostThreads) VGC_LAUNCH(kFew, 1024, 1);      // (by lane, of more than kFew / 2 rows a team)
            else if (L.rows_of_team > (uint32_t)kFew) VGC_LAUNCH(2 * kFew, 512, 8);        // (by lane 1024 threads hold these)
            else if (by_lane(A)) VGC_ROWS(1);
            else VGC_ROWS(8);
#undef VGC_ROWS
#undef VGC_LAUNCH
            return hip_check(hipGetLastError(), "launch k_group_norm_backward");
        });
    return by_samples(all, sizeof(T), L, [&](GroupNormArgs A, uint32_t B) {
        const dim3 grid(B * L.blocks * L.chunks);
#define VGC_LAUNCH(SUMS) do { \
        if (by_lane(A)) hipLaunchKernelGGL((k_group_norm_backward_rows<T, true, 1, SUMS>), grid, dim3(256), 0, stream, A); \
        else if (A.C % 8u == 0u) hipLaunchKernelGGL((k_group_norm_backward_rows<T, true, 8, SUMS>), grid, dim3(256), 0, stream, A); \
        else hipLaunchKernelGGL((k_group_norm_backward_rows<T, false, 8, SUMS>), grid, dim3(256), 0, stream, A); } while (0)
        VGC_LAUNCH(true);
        int rc = hip_check(hipGetLastError(), "launch k_group_norm_backward_rows");
        if (rc != VGC_OK) return rc;
        hipLaunchKernelGGL(k_group_norm_backward_join, dim3(B * A.G), dim3(join_threads(L, A.w)), 0, stream, A);
        if ((rc = hip_check(hipGetLastError(), "launch k_group_norm_backward_join")) != VGC_OK) return rc;
        VGC_LAUNCH(false);
#undef VGC_LAUNCH
        return hip_check(hipGetLastError(), "launch k_group_norm_backward_rows");
    });
}

int launch_group_norm_backward(int dtype, const void* dy, const void* x, const float* mean, const float* rstd, const float* gamma, const float* beta,
                               int act, uint32_t B, uint32_t P, uint32_t C, uint32_t G, float c, void* dx, float* g_gamma, float* s_gamma, float* g_beta,
                               float* s_beta, void* workspace, hipStream_t stream) {
    const GroupNormPlan L = group_norm_plan(dtype, true, B, P, C, G);
    const GroupNormSpace S = group_norm_space(L, B, C, G, true);
    char* ws = static_cast<char*>(workspace);
    GroupNormArgs A = {};
    A.x = x; A.dy = dy; A.gamma = gamma; A.beta = beta; A.mean = mean; A.rstd = rstd; A.out = dx;
    A.chunk_sums = (float*)(ws + S.chunk_sums);
    A.sums = (float*)(ws + S.sums);
    if (!L.held) A.group_sums = (float*)(ws + S.group_sums);
    A.B = B; A.P = P; A.C = C; A.G = G; A.w = C / G; A.act = (uint32_t)act;
    place(A, L);
    A.past = past_caches(dx, C, (uint64_t)B * P * C * (dtype == VGC_F32 ? 4u : 2u) * 3u);
    const int rc = dtype == VGC_F32 ? launch_group_norm_backward_of<float>(A, L, stream) : launch_group_norm_backward_of<uint16_t>(A, L, stream);
    if (rc != VGC_OK) return rc;
    return launch_column_sums(A.sums, 2, 0, B, 1, C, false, c, g_gamma, s_gamma, g_beta, s_beta, stream);
}

}  // namespace vgc
