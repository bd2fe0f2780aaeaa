// Layer norm over rows of C channels, forward and backward, with the sums over the samples of the scale's and the shift's
// gradients (Alg. 1, first two lines of the loop body, for those two vectors):
//   forward   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),  xhat = (x - mean) rstd,  y = gamma xhat + beta
//   backward  d = dy gamma,  dx = rstd (d - sum d / C - xhat sum (d xhat) / C)
//             sample z's gradients  G_z = sum_p dy xhat  and  H_z = sum_p dy;  g = c sum_z G_z,  s = c^2 sum_z G_z^2, H likewise
// Everything is float32 between the loads and the stores; the sum of squares is taken of the centred row, which is in
// registers by then, so that a large mean costs no digits.
//
// Both are bound by memory: x, y once forward; dy, x (or its 8-bit form) and dx once backward.  A row belongs to a team of
// lanes that hold it in registers, eight consecutive elements a lane and piece.  Backward, a team keeps its columns from row to
// row, so that the column sums stay in registers too and leave once per team, as float32 partial sums that a second, small
// kernel adds in a fixed order and, where a sample was spread over several teams, squares.  No atomics: results do not depend
// on scheduling.
#include <algorithm>

#include "vgc_rows.h"

namespace vgc {

// Sums of `kN` values over the lanes of a team, the same in all of them.  A team is a wave, or the whole workgroup; then `sh`
// holds a value per wave, and one barrier separates its writers from its readers (the caller alternates between two arrays).
template <int kN, bool kWide>
__device__ __forceinline__ void team_sums(float (&v)[kN], float (*sh)[kN], uint32_t waves) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = wave_sum(v[i]);
    if (kWide) {
        const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < kN; ++i) sh[wave][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = 0.f;
        for (uint32_t w = 0; w < waves; ++w)
#pragma unroll
            for (int i = 0; i < kN; ++i) v[i] += sh[w][i];
    }
}

constexpr uint32_t kMaxWaves = 16;

// The 8-bit form of the normalised piece (all lanes of the quad that holds the block take part).
__device__ __forceinline__ void keep_act8(const float (&f)[8], uint32_t C, uint32_t piece, uint64_t row, int n, int8_t* codes, uint8_t* exps) {
    const uint32_t field = act8_field(four_lanes_max(act8_top(f)));
    if (n <= 0) return;
    store_codes(codes + row * C + piece * 8u, act8_codes(f, field), n);
    if ((piece & 3u) == 0) exps[row * ((C + kAct8Block - 1) / kAct8Block) + piece / 4u] = (uint8_t)field;
}

// ---- forward --------------------------------------------------------------------------------------------------------------
// A team takes rows team, team + teams, ..: its part of gamma and beta stays in registers, and the next row is on its way while the
// present one is reduced and stored.  Teams: the waves of a workgroup (kWide false), or the workgroup.  (A row a workgroup, gamma and
// beta read for each: 16384 x 4096 bfloat16 with the 8-bit form 82 us; so 66.)
template <typename T, int kNV, bool kWide, bool kKeep>
__global__ __launch_bounds__(kWide ? 512 : 256) void k_layer_norm(const T* __restrict__ x, uint32_t R, uint32_t C, uint32_t teams, const float* __restrict__ gamma,
                                                                const float* __restrict__ beta, float eps, T* __restrict__ y,
                                                                float* __restrict__ mean_out, float* __restrict__ rstd_out,
                                                                int8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
    __shared__ float sh[2][kMaxWaves][1];
    const uint32_t lanes = kWide ? blockDim.x : 64u, lane = kWide ? threadIdx.x : threadIdx.x & 63u, waves = lanes / 64u;
    uint32_t row = kWide ? blockIdx.x : __builtin_amdgcn_readfirstlane(blockIdx.x * 4u + (threadIdx.x >> 6));
    if (row >= R) return;                                    // (a wave, or the workgroup)
    const float inv = 1.0f / (float)C;
    int n[kNV];
    Raw8<T> raw[kNV];
    float ga[kNV][8], be[kNV][8];
    auto request = [&](uint32_t r) {
#pragma unroll
        for (int i = 0; i < kNV; ++i) raw[i] = load8(x + (uint64_t)r * C + (lane + i * lanes) * 8u, n[i]);
    };
#pragma unroll
    for (int i = 0; i < kNV; ++i) n[i] = (int)C - (int)((lane + i * lanes) * 8u);
    request(row);
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        widen8(load8(gamma + (lane + i * lanes) * 8u, n[i]), ga[i]);
        widen8(load8(beta + (lane + i * lanes) * 8u, n[i]), be[i]);
    }
    for (;;) {
        float f[kNV][8], v[1] = {0.f};
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            widen8(raw[i], f[i]);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[0] += f[i][k];
        }
        const uint32_t after = row + teams;
        if (after < R) request(after);
        team_sums<1, kWide>(v, sh[0], waves);
        const float mean = v[0] * inv;
        v[0] = 0.f;
#pragma unroll
        for (int i = 0; i < kNV; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) {                    // elements past the row's end stay 0
                f[i][k] = k < n[i] ? f[i][k] - mean : 0.f;
                v[0] = __builtin_fmaf(f[i][k], f[i][k], v[0]);
            }
        team_sums<1, kWide>(v, sh[1], waves);
        const float rstd = 1.0f / sqrtf(v[0] * inv + eps);
        if (lane == 0) { mean_out[row] = mean; rstd_out[row] = rstd; }
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[i][k] *= rstd;
            if (kKeep) keep_act8(f[i], C, lane + i * lanes, row, n[i], codes, exps);
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = __builtin_fmaf(f[i][k], ga[i][k], be[i][k]);
            store8(y + (uint64_t)row * C + (lane + i * lanes) * 8u, o, n[i]);
        }
        if (after >= R) return;
        row = after;
    }
}

// Rows beyond what a team holds: a workgroup a row, read three times (the last two from the cache).
template <typename T, bool kKeep>
__global__ __launch_bounds__(1024) void k_layer_norm_long(const T* __restrict__ x, uint32_t C, const float* __restrict__ gamma,
                                                          const float* __restrict__ beta, float eps, T* __restrict__ y,
                                                          float* __restrict__ mean_out, float* __restrict__ rstd_out,
                                                          int8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
    __shared__ float sh[2][kMaxWaves][1];
    const uint32_t lanes = blockDim.x, lane = threadIdx.x, row = blockIdx.x;
    const T* xr = x + (uint64_t)row * C;
    const float inv = 1.0f / (float)C;
    float f[8], v[1] = {0.f};
    for (uint32_t e = lane * 8u; e < C; e += lanes * 8u) {
        widen8(load8(xr + e, (int)(C - e)), f);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[0] += f[k];
    }
    team_sums<1, true>(v, sh[0], lanes / 64u);
    const float mean = v[0] * inv;
    v[0] = 0.f;
    auto centred = [&](uint32_t e) {
        const int n = (int)C - (int)e;
        widen8(load8(xr + e, n), f);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = k < n ? f[k] - mean : 0.f;
    };
    for (uint32_t e = lane * 8u; e < C; e += lanes * 8u) {
        centred(e);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[0] = __builtin_fmaf(f[k], f[k], v[0]);
    }
    team_sums<1, true>(v, sh[1], lanes / 64u);
    const float rstd = 1.0f / sqrtf(v[0] * inv + eps);
    if (lane == 0) { mean_out[row] = mean; rstd_out[row] = rstd; }
    const uint32_t pieces = ((C + 31u) / 32u) * 4u;          // whole blocks: the lanes of one meet in keep_act8
    for (uint32_t p = lane; p < pieces; p += lanes) {
        const int n = (int)C - (int)(p * 8u);
        centred(p * 8u);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] *= rstd;
        if (kKeep) keep_act8(f, C, p, row, n, codes, exps);
        float ga[8], be[8], o[8];
        widen8(load8(gamma + p * 8u, n), ga);
        widen8(load8(beta + p * 8u, n), be);
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = __builtin_fmaf(f[k], ga[k], be[k]);
        store8(y + (uint64_t)row * C + p * 8u, o, n);
    }
}

// ---- backward -------------------------------------------------------------------------------------------------------------
// What the two forms of the normalised row need from memory: the row itself with its mean, or its 8-bit form.
template <typename T, bool kKept> struct RowIn;
template <typename T> struct RowIn<T, false> { Raw8<T> x; };
template <typename T> struct RowIn<T, true> { any_u2 q; uint32_t field; };

struct NormArgs {
    const void *dy, *x;
    const float *mean, *rstd, *gamma;
    const int8_t* codes;
    const uint8_t* exps;
    void* dx;
    float* partial;           // of team t: planes of C floats, see below
    uint32_t B, P, C, parts;  // teams a sample is spread over (1: a team takes whole samples)
    uint32_t teams;
};

template <typename T, bool kKept>
__device__ __forceinline__ RowIn<T, kKept> row_load(const NormArgs& A, uint64_t row, uint32_t piece, int n) {
    RowIn<T, kKept> r;
    if constexpr (kKept) {
        r.q = load_codes(A.codes + row * A.C + piece * 8u, n);
        r.field = n > 0 ? A.exps[row * ((A.C + kAct8Block - 1) / kAct8Block) + piece / 4u] : 0u;
    } else {
        r.x = load8(static_cast<const T*>(A.x) + row * A.C + piece * 8u, n);
    }
    return r;
}
template <typename T, bool kKept>
__device__ __forceinline__ void row_xhat(const RowIn<T, kKept>& r, float mean, float rstd, int n, float (&f)[8]) {
    if constexpr (kKept) {
        act8_values(r.q, r.field, f);
    } else {
        widen8(r.x, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = k < n ? (f[k] - mean) * rstd : 0.f;
    }
}

// Teams: the waves of a workgroup (kWide false), or the workgroup.  kRows rows are in flight at a time, the next ones' loads
// issued before the present ones are reduced.  kWhole: the team takes samples [t B / teams, (t + 1) B / teams) whole, keeps
// g and s of its columns, and leaves four planes (g and s of gamma, of beta); else it takes part t % parts of sample
// t / parts and leaves its two column sums.
template <typename T, bool kKept, int kNV, int kRows, bool kWide, bool kWhole>
__global__ __launch_bounds__(kWide ? 512 : 256) void k_layer_norm_backward(NormArgs A) {
    __shared__ float sh[2][kMaxWaves][2 * kRows];
    const uint32_t lanes = kWide ? blockDim.x : 64u, lane = kWide ? threadIdx.x : threadIdx.x & 63u, waves = lanes / 64u;
    const uint32_t team = kWide ? blockIdx.x : __builtin_amdgcn_readfirstlane(blockIdx.x * 4u + (threadIdx.x >> 6));
    if (team >= A.teams) return;                             // (a wave, or the workgroup)
    const uint32_t C = A.C, P = A.P;
    const float inv = 1.0f / (float)C;
    uint32_t row, end;                                       // the team's rows
    if (kWhole) {
        row = (uint32_t)((uint64_t)team * A.B / A.teams) * P;
        end = (uint32_t)((uint64_t)(team + 1u) * A.B / A.teams) * P;
    } else {
        const uint32_t z = team / A.parts, part = team - z * A.parts;
        row = z * P + (uint32_t)((uint64_t)part * P / A.parts);
        end = z * P + (uint32_t)((uint64_t)(part + 1u) * P / A.parts);
    }
    float ga[kNV][8];
    int n[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        n[i] = (int)C - (int)((lane + i * lanes) * 8u);
        widen8(load8(A.gamma + (lane + i * lanes) * 8u, n[i]), ga[i]);
    }
    constexpr int kS = kWhole ? kNV : 1;
    float cg[kNV][8] = {}, cb[kNV][8] = {};                  // column sums of the sample (or of its part)
    float gg[kS][8] = {}, gs[kS][8] = {}, bg[kS][8] = {}, bs[kS][8] = {};
    Raw8<T> dy[kRows][kNV];
    RowIn<T, kKept> in[kRows][kNV];
    float mean[kRows], rstd[kRows];
    auto request = [&](uint32_t at) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const uint64_t q = min(at + (uint32_t)r, end - 1u);          // (rows past the end are the last one again, and not used)
#pragma unroll
            for (int i = 0; i < kNV; ++i) {
                dy[r][i] = load8(static_cast<const T*>(A.dy) + q * C + (lane + i * lanes) * 8u, n[i]);
                in[r][i] = row_load<T, kKept>(A, q, lane + i * lanes, n[i]);
            }
            mean[r] = kKept ? 0.f : A.mean[q];
            rstd[r] = A.rstd[q];
        }
    };
    uint32_t turn = 0, left = P;                             // rows until the sample is complete
    if (row < end) request(row);
    for (; row < end; row += kRows) {
        float d[kRows][kNV][8], h[kRows][kNV][8], rs[kRows], v[2 * kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            rs[r] = rstd[r];
            float a = 0.f, b = 0.f;
            const float live = row + (uint32_t)r < end ? 1.f : 0.f;
#pragma unroll
            for (int i = 0; i < kNV; ++i) {
                widen8(dy[r][i], d[r][i]);
                row_xhat<T, kKept>(in[r][i], mean[r], rstd[r], n[i], h[r][i]);
                if (live != 0.f) {                           // (uniform)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        cb[i][k] += d[r][i][k];
                        cg[i][k] = __builtin_fmaf(d[r][i][k], h[r][i][k], cg[i][k]);
                    }
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    d[r][i][k] *= ga[i][k];
                    a += d[r][i][k];
                    b = __builtin_fmaf(d[r][i][k], h[r][i][k], b);
                }
            }
            v[2 * r] = a;
            v[2 * r + 1] = b;
            if (kWhole && live != 0.f && --left == 0) {      // square the sample's sums into s, add them into g, clear
                left = P;
#pragma unroll
                for (int i = 0; i < kS; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        gg[i][k] += cg[i][k];
                        gs[i][k] = __builtin_fmaf(cg[i][k], cg[i][k], gs[i][k]);
                        bg[i][k] += cb[i][k];
                        bs[i][k] = __builtin_fmaf(cb[i][k], cb[i][k], bs[i][k]);
                        cg[i][k] = cb[i][k] = 0.f;
                    }
            }
        }
        if (row + kRows < end) request(row + kRows);
        team_sums<2 * kRows, kWide>(v, sh[turn], waves);
        turn ^= 1u;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (row + (uint32_t)r >= end) break;
            const float a = v[2 * r] * inv, b = v[2 * r + 1] * inv;
            T* out = static_cast<T*>(A.dx) + (uint64_t)(row + (uint32_t)r) * C;
#pragma unroll
            for (int i = 0; i < kNV; ++i) {
                float o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = rs[r] * __builtin_fmaf(-h[r][i][k], b, d[r][i][k] - a);
                store8(out + (lane + i * lanes) * 8u, o, n[i]);
            }
        }
    }
    float* out = A.partial + (size_t)team * (kWhole ? 4u : 2u) * C;
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        const uint32_t e = (lane + i * lanes) * 8u;
        if (kWhole) {
            store8(out + e, gg[i < kS ? i : 0], n[i]);
            store8(out + C + e, gs[i < kS ? i : 0], n[i]);
            store8(out + 2 * (size_t)C + e, bg[i < kS ? i : 0], n[i]);
            store8(out + 3 * (size_t)C + e, bs[i < kS ? i : 0], n[i]);
        } else {
            store8(out + e, cg[i], n[i]);
            store8(out + C + e, cb[i], n[i]);
        }
    }
}

// Rows beyond what the largest workgroup holds: a workgroup per part of a sample, as above, that reads its rows twice (the
// second time from the cache) and keeps its column sums where they end up, in its own planes of the workspace.
template <typename T, bool kKept>
__global__ __launch_bounds__(1024) void k_layer_norm_backward_long(NormArgs A) {
    __shared__ float sh[2][kMaxWaves][2];
    const uint32_t lanes = blockDim.x, lane = threadIdx.x, team = blockIdx.x, C = A.C;
    const float inv = 1.0f / (float)C;
    const uint32_t z = team / A.parts, part = team % A.parts;
    const uint32_t p0 = (uint32_t)((uint64_t)part * A.P / A.parts), p1 = (uint32_t)((uint64_t)(part + 1u) * A.P / A.parts);
    float *cg = A.partial + (size_t)team * 2u * C, *cb = cg + C;
    uint32_t turn = 0;
    for (uint32_t p = p0; p < p1; ++p) {
        const uint64_t row = (uint64_t)z * A.P + p;
        const float mean = kKept ? 0.f : A.mean[row], rstd = A.rstd[row];
        float v[2] = {0.f, 0.f};
        for (int turns = 0; turns < 2; ++turns) {
            const float a = v[0] * inv, b = v[1] * inv;
            for (uint32_t e = lane * 8u; e < C; e += lanes * 8u) {
                const int n = (int)(C - e);
                float d[8], h[8], ga[8], o[8];
                widen8(load8(static_cast<const T*>(A.dy) + row * C + e, n), d);
                row_xhat<T, kKept>(row_load<T, kKept>(A, row, e / 8u, n), mean, rstd, n, h);
                widen8(load8(A.gamma + e, n), ga);
                if (turns == 0) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        v[0] += d[k] * ga[k];
                        v[1] = __builtin_fmaf(d[k] * ga[k], h[k], v[1]);
                    }
                    continue;
                }
                float sg[8] = {}, sb[8] = {};                // a lane's own columns: written before by this lane only
                if (p != p0) { widen8(load8(cg + e, n), sg); widen8(load8(cb + e, n), sb); }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    sg[k] = __builtin_fmaf(d[k], h[k], sg[k]);
                    sb[k] += d[k];
                    o[k] = rstd * __builtin_fmaf(-h[k], b, d[k] * ga[k] - a);
                }
                store8(cg + e, sg, n);
                store8(cb + e, sb, n);
                store8(static_cast<T*>(A.dx) + row * C + e, o, n);
            }
            if (turns == 0) team_sums<2, true>(v, sh[turn], lanes / 64u);
        }
        turn ^= 1u;
    }
}

// Adds the teams' partial sums in a fixed order: a workgroup takes 64 columns of one of the two vectors (blockIdx.y: gamma, beta),
// four a lane, and its 64 groups of 16 lanes share the partial sums between them.
//   whole samples: planes g, s, summed over the teams.
//   parts: the parts of a sample are added before the square.  Groups take samples of their own if there are 64 or more; below,
//   several groups share a sample's parts.
__global__ __launch_bounds__(1024) void k_layer_norm_sums(const float* __restrict__ partial, uint32_t teams, uint32_t B, uint32_t parts, uint32_t C,
                                                          int whole, float c, float* __restrict__ g_gamma, float* __restrict__ s_gamma,
                                                          float* __restrict__ g_beta, float* __restrict__ s_beta) {
    constexpr uint32_t kGroups = 64;
    __shared__ float sh[2][kGroups][64];
    const uint32_t lane = threadIdx.x & 15u, group = threadIdx.x >> 4, col = blockIdx.x * 64u + lane * 4u, vec = blockIdx.y;
    const int n = col < C ? (int)min(C - col, 4u) : 0;
    auto load = [&](const float* p) -> any_f4 {
        any_f4 r = {0.f, 0.f, 0.f, 0.f};
        if (n == 4) return *reinterpret_cast<const any_f4*>(p);
        for (int i = 0; i < 3; ++i)
            if (i < n) r[i] = p[i];
        return r;
    };
    any_f4 g = {0.f, 0.f, 0.f, 0.f}, s = g;
    uint32_t share = 1;                                      // groups a sample's parts are spread over
    if (whole) {
        const float* at = partial + (size_t)(2u * vec) * C + col;
        const size_t step = 4 * (size_t)C;
#pragma unroll 4
        for (uint32_t t = group; t < teams; t += kGroups) { g += load(at + t * step); s += load(at + t * step + C); }
    } else {
        const float* at = partial + (size_t)vec * C + col;
        const size_t step = 2 * (size_t)C;
        while (B * share * 2u <= kGroups) share *= 2u;
        const uint32_t sub = group % share;
        for (uint32_t z = group / share; z < B; z += kGroups / share) {
            any_f4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
            for (uint32_t q = sub; q < parts; q += share) sum += load(at + ((size_t)z * parts + q) * step);
            if (share > 1) { g = sum; break; }               // (at most one sample a group)
            g += sum;
            for (int i = 0; i < 4; ++i) s[i] = __builtin_fmaf(sum[i], sum[i], s[i]);
        }
    }
    for (int i = 0; i < 4; ++i) { sh[0][group][lane * 4u + i] = g[i]; sh[1][group][lane * 4u + i] = s[i]; }
    __syncthreads();
    // a thread takes one of the 64 columns and the sixteenth part of the groups, whole samples of them
    const uint32_t one = threadIdx.x & 63u, part = threadIdx.x >> 6;
    float go = 0.f, so = 0.f;
    if (share > 4u) {                                        // (fewer than 8 samples: each by one thread)
        if (part * share < kGroups) {
            float G = 0.f;
            for (uint32_t q = 0; q < share; ++q) G += sh[0][part * share + q][one];
            go = G;
            so = G * G;
        }
    } else {
        for (uint32_t q = 0; q < 4u; q += share) {
            float G = 0.f, S = 0.f;
            for (uint32_t e = 0; e < share; ++e) { G += sh[0][part * 4u + q + e][one]; S += sh[1][part * 4u + q + e][one]; }
            go += G;
            so += share > 1u ? G * G : S;
        }
    }
    __syncthreads();
    sh[0][part][one] = go;
    sh[1][part][one] = so;
    __syncthreads();
    const uint32_t at = blockIdx.x * 64u + one;
    if (part != 0u || at >= C) return;
    go = so = 0.f;
    for (uint32_t q = 0; q < 16u; ++q) { go += sh[0][q][one]; so += sh[1][q][one]; }
    float *gout = vec ? g_beta : g_gamma, *sout = vec ? s_beta : s_gamma;
    if (gout) gout[at] = c * go;
    sout[at] = c * c * so;
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
static uint32_t row_lanes(uint32_t C, uint32_t pieces_per_lane) { return ((C + 7) / 8 + pieces_per_lane * 64 - 1) / (pieces_per_lane * 64) * 64; }

int launch_layer_norm(int dtype, const void* x, uint64_t R, uint32_t C, const float* gamma, const float* beta, float eps, void* y, float* mean,
                      float* rstd, int8_t* codes, uint8_t* exps, hipStream_t stream) {
    if (R > 0x7FFFFFFFull) { set_error("vgc_layer_norm: %llu rows exceed the launch limit", (unsigned long long)R); return VGC_ERR_SIZE; }
    const uint32_t pieces = (C + 7) / 8, rows = (uint32_t)R;
    // Rows a wave holds are taken by waves, longer ones (up to 8192 elements) by workgroups; teams: four waves to a SIMD, which is what
    // the loads in flight need.  One piece a lane rather than two where a row has to itself what there is of the chip anyway.
    const bool one = pieces <= 64u || (rows <= 1024u && pieces > 64u && pieces <= 512u);
    const uint32_t lanes = row_lanes(C, one ? 1 : 2), teams = std::min(rows, 4096u / (lanes / 64u));
    const bool wide = lanes > 64u;
#define VGC_LAUNCH(T, NV, WIDE, KEEP) hipLaunchKernelGGL((k_layer_norm<T, NV, WIDE, KEEP>), dim3((WIDE) ? teams : (teams + 3) / 4), dim3((WIDE) ? lanes : 256u), 0, \
        stream, (const T*)x, rows, C, (WIDE) ? teams : (teams + 3) / 4 * 4, gamma, beta, eps, (T*)y, mean, rstd, codes, exps)
#define VGC_SHAPE(T, KEEP) do { \
        if (pieces > 1024u) hipLaunchKernelGGL((k_layer_norm_long<T, KEEP>), dim3(rows), dim3(1024), 0, stream, (const T*)x, C, gamma, beta, eps, (T*)y, mean, rstd, codes, exps); \
        else if (!wide) { if (one) VGC_LAUNCH(T, 1, false, KEEP); else VGC_LAUNCH(T, 2, false, KEEP); } \
        else { if (one) VGC_LAUNCH(T, 1, true, KEEP); else VGC_LAUNCH(T, 2, true, KEEP); } } while (0)
    if (dtype == VGC_F32) { if (codes) VGC_SHAPE(float, true); else VGC_SHAPE(float, false); }
    else { if (codes) VGC_SHAPE(uint16_t, true); else VGC_SHAPE(uint16_t, false); }
#undef VGC_SHAPE
#undef VGC_LAUNCH
    return hip_check(hipGetLastError(), "launch k_layer_norm");
}

struct NormTeams { uint32_t lanes, parts, teams; bool wide, whole, held; };
// About 2048 waves' worth of teams: two to a SIMD, which is what the loads in flight need.  Samples are taken whole when there
// are enough of them, else cut into parts of at least four rows.
static NormTeams norm_teams(uint32_t B, uint32_t P, uint32_t C) {
    NormTeams t;
    const uint32_t pieces = (C + 7) / 8;
    t.held = pieces <= 1024u;
    t.lanes = t.held ? row_lanes(C, pieces <= 64u ? 1 : 2) : 1024u;
    t.wide = t.lanes > 64u;
    const uint32_t want = 2048u / (t.lanes / 64u);
    t.whole = t.held && B >= want;
    if (t.whole) { t.parts = 1; t.teams = want; return t; }
    t.parts = std::min((want + B - 1) / B, (P + 3) / 4);
    t.teams = B * t.parts;
    return t;
}
size_t layer_norm_backward_workspace_bytes(uint32_t B, uint32_t P, uint32_t C) {
    const NormTeams t = norm_teams(B, P, C);
    return (size_t)t.teams * (t.whole ? 4u : 2u) * C * sizeof(float);
}

int launch_layer_norm_backward(int dtype, const void* dy, const void* x, const float* mean, const int8_t* codes, const uint8_t* exps,
                               const float* rstd, const float* gamma, uint32_t B, uint32_t P, uint32_t C, float c, void* dx, float* g_gamma,
                               float* s_gamma, float* g_beta, float* s_beta, void* workspace, hipStream_t stream) {
    const NormTeams t = norm_teams(B, P, C);
    const NormArgs A = {dy, x, mean, rstd, gamma, codes, exps, dx, static_cast<float*>(workspace), B, P, C, t.parts, t.teams};
    const dim3 grid(t.wide ? t.teams : (t.teams + 3) / 4), block(t.wide ? t.lanes : 256u);
    const uint32_t pieces = (C + 7) / 8;
#define VGC_LAUNCH(T, KEPT, NV, ROWS, WIDE, WHOLE) hipLaunchKernelGGL((k_layer_norm_backward<T, KEPT, NV, ROWS, WIDE, WHOLE>), grid, block, 0, stream, A)
#define VGC_SHAPE(T, KEPT) do { \
        if (!t.held) hipLaunchKernelGGL((k_layer_norm_backward_long<T, KEPT>), grid, block, 0, stream, A); \
        else if (pieces <= 64u) { if (t.whole) VGC_LAUNCH(T, KEPT, 1, 2, false, true); else VGC_LAUNCH(T, KEPT, 1, 2, false, false); } \
        else if (!t.wide) { if (t.whole) VGC_LAUNCH(T, KEPT, 2, 2, false, true); else VGC_LAUNCH(T, KEPT, 2, 2, false, false); } \
        else { if (t.whole) VGC_LAUNCH(T, KEPT, 2, 2, true, true); else VGC_LAUNCH(T, KEPT, 2, 2, true, false); } } while (0)
    if (dtype == VGC_F32) { if (codes) VGC_SHAPE(float, true); else VGC_SHAPE(float, false); }
    else { if (codes) VGC_SHAPE(uint16_t, true); else VGC_SHAPE(uint16_t, false); }
#undef VGC_SHAPE
#undef VGC_LAUNCH
    int rc = hip_check(hipGetLastError(), "launch k_layer_norm_backward");
    if (rc != VGC_OK) return rc;
    hipLaunchKernelGGL(k_layer_norm_sums, dim3((C + 63) / 64, 2), dim3(1024), 0, stream, (const float*)workspace, t.teams, B, t.parts, C, (int)t.whole,
                       c, g_gamma, s_gamma, g_beta, s_beta);
    return hip_check(hipGetLastError(), "launch k_layer_norm_sums");
}

}  // namespace vgc
