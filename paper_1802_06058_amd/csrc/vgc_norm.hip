// Layer norm over rows of C channels, forward and backward, with the sums over the samples of the scale's and the shift's
// gradients (Alg. 1, first two lines of the loop body, for those two vectors):
//   forward   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),  xhat = (x - mean) rstd,  y = gamma xhat + beta
//   backward  d = dy gamma,  dx = rstd (d - sum d / C - xhat sum (d xhat) / C)
//             sample z's gradients  G_z = sum_p dy xhat  and  H_z = sum_p dy;  g = c sum_z G_z,  s = c^2 sum_z G_z^2, H likewise
// Everything is float32 between the loads and the stores; the sum of squares is taken of the centred row, which is in
// registers by then, so that a large mean costs no digits.
//
// Both are bound by memory: x, y once forward; dy, x (or its 8-bit form) and dx once backward.  A row belongs to a team of
// 8, 16, 32 or 64 lanes, or to a workgroup, as it needs to hold it in registers, eight consecutive elements a lane and piece.
// Backward, a team keeps its columns from row to row, so that the column sums stay in registers too; they leave once per workgroup, as
// float32 partial sums that a second, small kernel adds in a fixed order and, where a sample was spread over several workgroups,
// squares.  No atomics: results do not depend on scheduling.
#include <algorithm>

#include "vgc_rows.h"

namespace vgc {

// Sums of `kN` values over the lanes of a team, the same in all of them: kL lanes, or (kL = 0) the workgroup.  Then `sh` holds a value
// per wave, and one barrier separates its writers from its readers (the caller alternates between two arrays).
template <int kN, int kL>
__device__ __forceinline__ void team_sums(float (&v)[kN], float (*sh)[kN], uint32_t waves) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = lanes_sum<kL == 0 ? 64 : kL>(v[i]);
    if (kL == 0) {
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
// present one is reduced and stored.  Teams: kL lanes each, or (kL = 0) the workgroup.  (A row a workgroup, gamma and beta read for each:
// 16384 x 4096 bfloat16 68.5 us; so 52.6.)
// 16384 x 4096 bfloat16: 50 us, 5.4 TB/s of x and y; kept in 8 bits too and decoded again by vgc_act8_decode 107, 5.0 TB/s.  128 x 1000
// float32: 8 us a call, which is the call's own time.
template <typename T, int kNV, int kL, bool kKeep>
__global__ __launch_bounds__(kL == 0 ? 512 : 256) void k_layer_norm(const T* __restrict__ x, uint32_t R, uint32_t C, uint32_t teams, const float* __restrict__ gamma,
                                                                const float* __restrict__ beta, float eps, T* __restrict__ y,
                                                                float* __restrict__ mean_out, float* __restrict__ rstd_out,
                                                                int8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
    __shared__ float sh[2][kMaxWaves][1];
    const uint32_t lanes = kL == 0 ? blockDim.x : (uint32_t)kL, lane = kL == 0 ? threadIdx.x : threadIdx.x % lanes, waves = lanes / 64u;
    uint32_t row = kL == 0 ? blockIdx.x : blockIdx.x * (256u / lanes) + threadIdx.x / lanes;
    if (row >= R) return;                                    // (a team)
    const float inv = 1.0f / (float)C;
    int n[kNV];
    Raw8<T> raw[kNV];
    float ga[kNV][8], be[kNV][8];
    auto request = [&](uint32_t r) {
#pragma unroll
        for (int i = 0; i < kNV; ++i) raw[i] = load8(x + (uint64_t)r * C + (lane + i * lanes) * 8u, n[i], rows_at_end(r, R));
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
            if (C % 8u != 0) clip8(raw[i], n[i]);
            widen8(raw[i], f[i]);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[0] += f[i][k];
        }
        const uint32_t after = row + teams;
        if (after < R) request(after);
        team_sums<1, kL>(v, sh[0], waves);
        const float mean = v[0] * inv;
        v[0] = 0.f;
#pragma unroll
        for (int i = 0; i < kNV; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) {                    // elements past the row's end stay 0
                f[i][k] = k < n[i] ? f[i][k] - mean : 0.f;
                v[0] = __builtin_fmaf(f[i][k], f[i][k], v[0]);
            }
        team_sums<1, kL>(v, sh[1], waves);
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

// Rows beyond what a team holds: a workgroup a row, read three times (the last two from the cache).  16384 x 12288 bfloat16: 219 us, 3.7 TB/s of x
// and y, bound by the three passes following each other.
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
    team_sums<1, 0>(v, sh[0], lanes / 64u);
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
    team_sums<1, 0>(v, sh[1], lanes / 64u);
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
    float* partial;           // of every workgroup: planes of C floats, see below
    uint32_t B, P, C, parts;  // workgroups a sample is spread over
    uint32_t groups;
};

template <typename T, bool kKept>
__device__ __forceinline__ RowIn<T, kKept> row_load(const NormArgs& A, uint64_t row, uint32_t piece, int n, bool at_end) {
    RowIn<T, kKept> r;
    if constexpr (kKept) {
        r.q = load_codes(A.codes + row * A.C + piece * 8u, n, at_end);
        r.field = n > 0 ? A.exps[row * ((A.C + kAct8Block - 1) / kAct8Block) + piece / 4u] : 0u;
    } else {
        r.x = load8(static_cast<const T*>(A.x) + row * A.C + piece * 8u, n, at_end);
    }
    return r;
}
template <typename T, bool kKept>
__device__ __forceinline__ void row_xhat(RowIn<T, kKept>& r, float mean, float rstd, int n, bool ragged, float (&f)[8]) {
    if constexpr (kKept) {
        if (ragged) clip_codes(r.q, n);
        act8_values(r.q, r.field, f);
    } else {
        widen8(r.x, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = k < n ? (f[k] - mean) * rstd : 0.f;
    }
}

// Teams: kL lanes each, or (kL = 0) the workgroup.  kRows rows are in flight at a time, the next ones' loads issued before the
// present ones are reduced.  kWhole: a team takes samples whole, number t of n teams those of [t B / n, (t + 1) B / n), and keeps g
// and s of its columns; the workgroup leaves four planes (g and s of gamma, of beta), its teams' added.  Else a workgroup takes part
// w % parts of sample w / parts, its teams rows in turn, and leaves its two column sums.  Bound by memory: 16 samples of 1024 x 4096
// bfloat16 from the kept rows 72 us with the sums, 4.7 TB/s of dy, codes and dx; 32 of 49 x 2048 float32 from x 15.7, of which 8 are the call's.
template <typename T, bool kKept, int kNV, int kRows, int kL, bool kWhole>
__global__ __launch_bounds__(kL == 0 ? 512 : 256) void k_layer_norm_backward(NormArgs A) {
    constexpr uint32_t kTeams = kL == 0 ? 1u : 256u / (kL == 0 ? 1 : kL);
    __shared__ float sh[2][kMaxWaves][2 * kRows];
    __shared__ float add[kL == 0 ? 1 : 256 * kNV * 8];
    const uint32_t lanes = kL == 0 ? blockDim.x : (uint32_t)kL, lane = kL == 0 ? threadIdx.x : threadIdx.x % lanes, waves = lanes / 64u;
    const uint32_t team = kL == 0 ? 0u : threadIdx.x / lanes, C = A.C, P = A.P;
    const float inv = 1.0f / (float)C;
    const uint64_t rows = (uint64_t)A.B * P;
    const bool ragged = C % 8u != 0;                         // (a row's last piece is short)
    uint32_t row, end, step;                                 // the team's rows
    if (kWhole) {
        const uint64_t t = (uint64_t)blockIdx.x * kTeams + team, n = (uint64_t)A.groups * kTeams;
        row = (uint32_t)(t * A.B / n) * P;
        end = (uint32_t)((t + 1u) * A.B / n) * P;
        step = 1u;
    } else {
        const uint32_t z = blockIdx.x / A.parts, part = blockIdx.x - z * A.parts;
        row = z * P + (uint32_t)((uint64_t)part * P / A.parts) + team;
        end = z * P + (uint32_t)((uint64_t)(part + 1u) * P / A.parts);
        step = kTeams;
    }
    float ga[kNV][8];
    int n[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        n[i] = (int)C - (int)((lane + i * lanes) * 8u);
        widen8(load8(A.gamma + (lane + i * lanes) * 8u, n[i]), ga[i]);
    }
    constexpr int kS = kWhole ? kNV : 1;
    float cg[kNV][8] = {}, cb[kNV][8] = {};                  // column sums of the sample (or of the team's rows of it)
    float gg[kS][8] = {}, gs[kS][8] = {}, bg[kS][8] = {}, bs[kS][8] = {};
    Raw8<T> dy[kRows][kNV];
    RowIn<T, kKept> in[kRows][kNV];
    float mean[kRows], rstd[kRows];
    auto request = [&](uint32_t at) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const uint64_t q = at + r * step < end ? at + r * step : at;   // (rows past the end are the first one again, and not used)
#pragma unroll
            for (int i = 0; i < kNV; ++i) {
                dy[r][i] = load8(static_cast<const T*>(A.dy) + q * C + (lane + i * lanes) * 8u, n[i], rows_at_end(q, rows));
                in[r][i] = row_load<T, kKept>(A, q, lane + i * lanes, n[i], rows_at_end(q, rows));
            }
            mean[r] = kKept ? 0.f : A.mean[q];
            rstd[r] = A.rstd[q];
        }
    };
    uint32_t turn = 0, left = P;                             // rows until the sample is complete
    if (row < end) request(row);
    for (; row < end; row += kRows * step) {
        float d[kRows][kNV][8], h[kRows][kNV][8], rs[kRows], v[2 * kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            rs[r] = rstd[r];
            float a = 0.f, b = 0.f;
            const bool live = row + r * step < end;
#pragma unroll
            for (int i = 0; i < kNV; ++i) {
                if (ragged) clip8(dy[r][i], n[i]);
                widen8(dy[r][i], d[r][i]);
                row_xhat<T, kKept>(in[r][i], mean[r], rstd[r], n[i], ragged, h[r][i]);
                if (live) {                                  // (the same in a team)
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
            if (kWhole && live && --left == 0) {             // square the sample's sums into s, add them into g, clear
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
        if (row + kRows * step < end) request(row + kRows * step);
        team_sums<2 * kRows, kL>(v, sh[turn], waves);
        turn ^= 1u;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (row + r * step >= end) break;
            const float a = v[2 * r] * inv, b = v[2 * r + 1] * inv;
            T* out = static_cast<T*>(A.dx) + (uint64_t)(row + r * step) * C;
#pragma unroll
            for (int i = 0; i < kNV; ++i) {
                float o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = rs[r] * __builtin_fmaf(-h[r][i][k], b, d[r][i][k] - a);
                store8(out + (lane + i * lanes) * 8u, o, n[i]);
            }
        }
    }
    float* out = A.partial + (size_t)blockIdx.x * (kWhole ? 4u : 2u) * C;
    auto leave = [&](const float (&x)[kNV][8], uint32_t plane) {           // the teams' sums in order, by the first team
        float sum[kNV][8];
#pragma unroll
        for (int i = 0; i < kNV; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[i][k] = x[i][k];
        if (kL != 0) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kNV; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) add[(i * 8 + k) * 256u + threadIdx.x] = x[i][k];
            __syncthreads();
            if (team != 0u) return;
            for (uint32_t t = 1; t < kTeams; ++t)
#pragma unroll
                for (int i = 0; i < kNV; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[i][k] += add[(i * 8 + k) * 256u + t * lanes + lane];
        }
#pragma unroll
        for (int i = 0; i < kNV; ++i) store8(out + (size_t)plane * C + (lane + i * lanes) * 8u, sum[i], n[i]);
    };
    if constexpr (kWhole) {
        leave(gg, 0);
        leave(gs, 1);
        leave(bg, 2);
        leave(bs, 3);
    } else {
        leave(cg, 0);
        leave(cb, 1);
    }
}

// Rows beyond what the largest workgroup holds: a workgroup per part of a sample, as above, that reads its rows twice (the
// second time from the cache) and keeps its column sums where they end up, in its own planes of the workspace.  16 x 1024 x 12288 bfloat16 from
// x: 804 us, 1.5 TB/s of dy, x and dx: the column sums are read and written for every row.
template <typename T, bool kKept>
__global__ __launch_bounds__(1024) void k_layer_norm_backward_long(NormArgs A) {
    __shared__ float sh[2][kMaxWaves][2];
    const uint32_t lanes = blockDim.x, lane = threadIdx.x, C = A.C;
    const float inv = 1.0f / (float)C;
    const uint32_t z = blockIdx.x / A.parts, part = blockIdx.x % A.parts;
    const uint32_t p0 = (uint32_t)((uint64_t)part * A.P / A.parts), p1 = (uint32_t)((uint64_t)(part + 1u) * A.P / A.parts);
    float *cg = A.partial + (size_t)blockIdx.x * 2u * C, *cb = cg + C;
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
                RowIn<T, kKept> in = row_load<T, kKept>(A, row, e / 8u, n, true);
                row_xhat<T, kKept>(in, mean, rstd, n, false, h);
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
            if (turns == 0) team_sums<2, 0>(v, sh[turn], lanes / 64u);
        }
        turn ^= 1u;
    }
}

// Adds the teams' partial sums in a fixed order: a workgroup takes 64 columns of one of the two vectors (blockIdx.y: gamma, beta),
// four a lane, and its 64 groups of 16 lanes share the partial sums between them.
//   vecs: vectors a group of partial sums holds, one after another.
//   whole samples: planes g, s, summed over the workgroups that left them.
//   parts: the parts of a sample are added before the square.  Groups take samples of their own if there are 64 or more; below,
//   several groups share a sample's parts.
__global__ __launch_bounds__(1024) void k_layer_norm_sums(const float* __restrict__ partial, uint32_t vecs, uint32_t groups, uint32_t B, uint32_t parts, uint32_t C,
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
        const size_t step = 2 * (size_t)vecs * C;
#pragma unroll 4
        for (uint32_t t = group; t < groups; t += kGroups) { g += load(at + t * step); s += load(at + t * step + C); }
    } else {
        const float* at = partial + (size_t)vec * C + col;
        const size_t step = (size_t)vecs * C;
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
// A team: the fewest lanes (8, 16, 32, 64) that hold a row with a piece each, 64 with two pieces (forward only: backward, a lane has one up to
// 4096 elements), or a workgroup (`group`) of as many waves as it takes with two pieces a lane (with one: `single`).  held: rows of up to
// 8192 elements.
struct Team { uint32_t lanes; bool group, single, held; };
static Team team_of(uint32_t C, bool single) {
    const uint32_t pieces = (C + 7) / 8, each = single ? 64u : 128u;
    Team t = {64u, pieces > each, single, pieces <= 1024u};
    if (t.group) t.lanes = t.held ? (pieces + each - 1) / each * 64u : 1024u;
    else if (pieces <= 64u) { t.single = true; t.lanes = pieces <= 8u ? 8u : pieces <= 16u ? 16u : pieces <= 32u ? 32u : 64u; }
    return t;
}

// 2^16 rows a launch: 2^22 workgroups would have 2^32 threads, which no launch has.  (The kernel with a loop over rows: 16384 x 12288 bfloat16
// 220 -> 240 us.)
template <typename T, bool kKeep>
static void launch_layer_norm_long(const void* x, uint32_t rows, uint32_t C, const float* gamma, const float* beta, float eps, void* y, float* mean, float* rstd,
                                   int8_t* codes, uint8_t* exps, hipStream_t stream) {
    for (uint32_t r = 0; r < rows; r += 1u << 16) {
        const size_t at = (size_t)r * C;
        hipLaunchKernelGGL((k_layer_norm_long<T, kKeep>), dim3(std::min(rows - r, 1u << 16)), dim3(1024), 0, stream, (const T*)x + at, C, gamma, beta, eps, (T*)y + at,
                           mean + r, rstd + r, kKeep ? codes + at : nullptr, kKeep ? exps + (size_t)r * ((C + kAct8Block - 1) / kAct8Block) : nullptr);
    }
}

int launch_layer_norm(int dtype, const void* x, uint64_t R, uint32_t C, const float* gamma, const float* beta, float eps, void* y, float* mean,
                      float* rstd, int8_t* codes, uint8_t* exps, hipStream_t stream) {
    if (R > 0x7FFFFFFFull) { set_error("vgc_layer_norm: %llu rows exceed the launch limit", (unsigned long long)R); return VGC_ERR_SIZE; }
    // Sixteen waves a compute unit, which is what the loads in flight need, in whole workgroups a compute unit.  Many rows that are not
    // kept: one piece a lane (us; bfloat16, two pieces and one: 16384 x 4096 52.6 and 49.9, 60000 x 2048 94.5 and 91.4, but 4096 x 4096 13.5
    // and 14.9, 16384 x 4096 kept 107.3 and 108.5; between 4096 and 16384 rows not measured).
    const uint32_t rows = (uint32_t)R;
    const Team t = team_of(C, !codes && rows >= 16384u && C <= 4096u);
    const uint32_t each = t.group ? 1u : 256u / t.lanes, want = 256u * (t.group ? std::max(1u, 16u / (t.lanes / 64u)) : 4u);
    const uint32_t groups = std::min((rows + each - 1) / each, want);
#define VGC_LAUNCH(T, NV, L, KEEP) hipLaunchKernelGGL((k_layer_norm<T, NV, L, KEEP>), dim3(groups), dim3(t.group ? t.lanes : 256u), 0, stream, \
        (const T*)x, rows, C, groups * each, gamma, beta, eps, (T*)y, mean, rstd, codes, exps)
#define VGC_SHAPE(T, KEEP) do { \
        if (!t.held) launch_layer_norm_long<T, KEEP>(x, rows, C, gamma, beta, eps, y, mean, rstd, codes, exps, stream); \
        else if (t.group && t.single) VGC_LAUNCH(T, 1, 0, false); \
        else if (t.group) VGC_LAUNCH(T, 2, 0, KEEP); \
        else if (!t.single) VGC_LAUNCH(T, 2, 64, KEEP); \
        else if (t.lanes == 64u) VGC_LAUNCH(T, 1, 64, KEEP); \
        else if (t.lanes == 32u) VGC_LAUNCH(T, 1, 32, KEEP); \
        else if (t.lanes == 16u) VGC_LAUNCH(T, 1, 16, KEEP); \
        else VGC_LAUNCH(T, 1, 8, KEEP); } while (0)
    if (dtype == VGC_F32) { if (codes) VGC_SHAPE(float, true); else VGC_SHAPE(float, false); }
    else { if (codes) VGC_SHAPE(uint16_t, true); else VGC_SHAPE(uint16_t, false); }
#undef VGC_SHAPE
#undef VGC_LAUNCH
    return hip_check(hipGetLastError(), "launch k_layer_norm");
}

struct NormPlan { Team team; uint32_t parts, groups; bool whole; };
// Workgroups come in multiples of the 256 compute units, or just below one: a few beyond it take as long as all of the next (48 samples of
// 1257 x 2500 kept rows: 432 workgroups of five waves 177 us, 624 of them 226).  As many times 256 as are resident, 16 waves a compute unit (8
// with two pieces a lane, 12 with whole samples; a workgroup's waves counted as a power of two, as they share out the SIMDs), while a
// team has 48 rows to go through for the partial sums it leaves (whole samples: 96); up to 8 waves a compute unit while it has 8.
// A sample is cut into parts of at least two rows a team (four for a workgroup); samples are taken whole where a team then has no more
// rows to go through, one after another (16384 samples of one row of 2048 bfloat16: whole 53 us, apart 317).
static NormPlan norm_plan(uint32_t B, uint32_t P, uint32_t C) {
    NormPlan L;
    L.team = team_of(C, C <= 4096u);                         // (one piece a lane: 60336 rows of 2048 bfloat16 176 -> 166 us, of 4096 367 -> 300)
    auto up = [](uint64_t a, uint64_t b) { return (a + b - 1) / b; };
    const uint32_t teams = L.team.group ? 1u : 256u / L.team.lanes, of = L.team.group ? L.team.lanes / 64u : 4u;
    const uint32_t waves = of <= 1u ? 1u : of == 2u ? 2u : of <= 4u ? 4u : of <= 8u ? 8u : 16u;
    auto times = [&](uint32_t resident, uint64_t rows) {     // workgroups a compute unit
        const uint64_t most = resident / waves, some = 8u / waves, each = (uint64_t)B * P / (teams * 256u);
        return (uint32_t)std::max<uint64_t>(1, std::max(std::min(most, each / rows), std::min(std::min(most, some), each / 8u)));
    };
    const uint32_t rows = L.team.group ? 4u : 2u * teams;    // of a part at least
    const uint32_t want = 256u * times(L.team.single ? 16u : 8u, 48u), want_whole = 256u * times(L.team.single ? 12u : 8u, 96u);
    L.parts = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(want / B, up(P, rows)));
    L.whole = L.team.held && P * up(B, (uint64_t)want_whole * teams) <= up(P, (uint64_t)teams * L.parts) * up((uint64_t)B * L.parts, want);
    if (L.whole) L.parts = 1;
    L.groups = L.whole ? (uint32_t)std::min<uint64_t>(up(B, teams), want_whole) : B * L.parts;
    return L;
}
size_t layer_norm_backward_workspace_bytes(uint32_t B, uint32_t P, uint32_t C) {
    const NormPlan L = norm_plan(B, P, C);
    return (size_t)L.groups * (L.whole ? 4u : 2u) * C * sizeof(float);
}

int launch_layer_norm_backward(int dtype, const void* dy, const void* x, const float* mean, const int8_t* codes, const uint8_t* exps,
                               const float* rstd, const float* gamma, uint32_t B, uint32_t P, uint32_t C, float c, void* dx, float* g_gamma,
                               float* s_gamma, float* g_beta, float* s_beta, void* workspace, hipStream_t stream) {
    const NormPlan L = norm_plan(B, P, C);
    const Team& t = L.team;
    const NormArgs A = {dy, x, mean, rstd, gamma, codes, exps, dx, static_cast<float*>(workspace), B, P, C, L.parts, L.groups};
    const dim3 grid(L.groups), block(t.group ? t.lanes : 256u);
    // (two rows in flight: 16 x 1024 x 4096 bfloat16 kept 72 us, with one 82; one where whole samples of two pieces a lane leave no registers
    // for two)
#define VGC_LAUNCH(T, KEPT, NV, LANES) do { \
        if (L.whole) hipLaunchKernelGGL((k_layer_norm_backward<T, KEPT, NV, NV == 2 ? 1 : 2, LANES, true>), grid, block, 0, stream, A); \
        else hipLaunchKernelGGL((k_layer_norm_backward<T, KEPT, NV, 2, LANES, false>), grid, block, 0, stream, A); } while (0)
#define VGC_SHAPE(T, KEPT) do { \
        if (!t.held) hipLaunchKernelGGL((k_layer_norm_backward_long<T, KEPT>), grid, block, 0, stream, A); \
        else if (t.group && t.single) VGC_LAUNCH(T, KEPT, 1, 0); \
        else if (t.group) VGC_LAUNCH(T, KEPT, 2, 0); \
        else if (t.lanes == 64u) VGC_LAUNCH(T, KEPT, 1, 64); \
        else if (t.lanes == 32u) VGC_LAUNCH(T, KEPT, 1, 32); \
        else if (t.lanes == 16u) VGC_LAUNCH(T, KEPT, 1, 16); \
        else VGC_LAUNCH(T, KEPT, 1, 8); } while (0)
    if (dtype == VGC_F32) { if (codes) VGC_SHAPE(float, true); else VGC_SHAPE(float, false); }
    else { if (codes) VGC_SHAPE(uint16_t, true); else VGC_SHAPE(uint16_t, false); }
#undef VGC_SHAPE
#undef VGC_LAUNCH
    int rc = hip_check(hipGetLastError(), "launch k_layer_norm_backward");
    if (rc != VGC_OK) return rc;
    return launch_column_sums((const float*)workspace, 2, L.groups, B, L.parts, C, L.whole, c, g_gamma, s_gamma, g_beta, s_beta, stream);
}

int launch_column_sums(const float* partial, uint32_t vecs, uint32_t groups, uint32_t B, uint32_t parts, uint32_t C, bool whole, float c, float* g0, float* s0,
                       float* g1, float* s1, hipStream_t stream) {
    hipLaunchKernelGGL(k_layer_norm_sums, dim3((C + 63) / 64, vecs), dim3(1024), 0, stream, partial, vecs, groups, B, parts, C, (int)whole, c, g0, s0, g1, s1);
    return hip_check(hipGetLastError(), "launch k_layer_norm_sums");
}

}  // namespace vgc
