// Softmax cross entropy of a linear layer over many classes, without its logits:
//   z[n, v] = sum_h X[n, h] W[v, h],   lse[n] = log sum_v exp z[n, v],   loss[n] = lse[n] - z[n, t_n]
//   backward  D[n, v] = w_n (exp(z[n, v] - lse[n]) - [v = t_n]),   dX = D W,
//             sample z's gradient of W  G_z = sum_p D[z, p, :]^T X[z, p, :],   g = c sum_z G_z,   s = c^2 sum_z G_z . G_z
//
// Forward, the logits of a tile stay in the accumulators: a token's column of them is reduced to its maximum and the sum of the
// exponentials relative to it, and these pairs are joined over the tiles of the vocabulary by a second, small kernel.  W is the A
// operand, so that a lane's 16 results of an instruction are 16 classes of one token: the reduction is in registers but for one
// exchange between the lane halves.
// Backward, the logits are formed again, a piece of the vocabulary at a time, and D of the piece goes to the workspace by classes,
// positions contiguous: the order in which the sums over a sample's positions read it with k contiguous and dX reads it with k, the
// classes, as rows, beside W as it lies.  Memory is bounded by the piece, not by the vocabulary.  The three products run through
// the loop of vgc_gemm.h.
//
// Precision.  bfloat16 inputs: products are exact, sums float32.  D, relative to its sample's largest weight, is rounded to bfloat16 for
// dX, which is rounded to bfloat16 itself; what that left of the target's entry, which all other classes' entries add up to, is added
// to dX in float (128 rows of 1024, 8192 classes, without: dX 2.04e-3 off, so 1.66e-3, which its own rounding alone is).  For g and s, which
// are float32, a second plane holds the rest, 16 significant bits in all, and for samples of few positions or small products a third what
// that leaves; samples of one position have D in float.  (A third plane for the target's entries alone was tried: k_loss_sums has no
// registers for it.)  float32 inputs: every operand is cut exactly into three planes of 8 bits, rounded, and a product is formed from the
// six pairs of planes that reach 2^-24 of it; few rows are multiplied as floats instead.
#include <algorithm>

#include "vgc_gemm.h"
#include "vgc_planes.h"

namespace vgc {

// ---- operands -------------------------------------------------------------------------------------------------------------
// Rows as they are, padded with zeros to whole pieces of 8; of one matrix or two, whose workgroups follow each other.
template <typename T>
__global__ __launch_bounds__(256) void k_planes_rows(PlaneRows first, PlaneRows second, uint32_t groups) {
    const bool other = blockIdx.x >= groups;
    const PlaneRows M = other ? second : first;
    const uint32_t Kp = (M.K + 7u) / 8u * 8u, per_row = Kp / 8u;
    const uint64_t i = (uint64_t)(blockIdx.x - (other ? groups : 0u)) * 256u + threadIdx.x;
    if (i >= (uint64_t)M.R * per_row) return;
    const uint64_t row = i / per_row;
    const uint32_t k = (uint32_t)(i - row * per_row) * 8u;
    float f[8];
    widen8(load8(static_cast<const T*>(M.src) + row * M.K + k, (int)(M.K - k)), f);
    store_planes<T>(M.dst + row * Kp + k, (uint64_t)M.R * Kp, f);
}

// Positions: sample z's position p is number z Pp + p, P <= Pp; the numbers between are no positions.
struct Positions {
    uint32_t B, P, Pp;
    __device__ __forceinline__ uint32_t row(uint32_t q) const {            // its row of [B, P], or ~0
        const uint32_t z = q / Pp, p = q - z * Pp;
        return z < B && p < P ? z * P + p : 0xFFFFFFFFu;
    }
};

// What D of a sample is relative to while it is rounded: with bfloat16 inputs its largest weight, so that the entry of a missed class,
// which is most of what g, s and dX consist of, is -1 in bfloat16 as it is, and not a weight's rounding that all positions of a
// sample share (2 x 38 positions, weights 1/38, 44209 classes: s 4.4e-6 off, so 2.1e-6).  of: by sample, or (own: samples of one position)
// the weights themselves; NULL: 1.
__device__ __forceinline__ float scale_from(float top) { return top > 0.f && top < __builtin_inff() ? top : 1.f; }
struct Scales {
    const float* of;
    bool own;
    __device__ __forceinline__ float at(uint32_t z) const { return !of ? 1.f : own ? scale_from(fabsf(of[z])) : of[z]; }
};
__global__ __launch_bounds__(1024) void k_loss_scales(const float* __restrict__ weight, const int64_t* __restrict__ target, uint32_t P, float* __restrict__ scales) {
    __shared__ float sh[16];
    float top = 0.f;
    for (uint32_t p = threadIdx.x; p < P; p += 1024u) {
        const size_t row = (size_t)blockIdx.x * P + p;
        if (target[row] >= 0) top = fmaxf(top, fabsf(weight[row]));
    }
    lanes_max<64>(top);
    if ((threadIdx.x & 63u) == 0u) sh[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x != 0u) return;
    for (int w = 1; w < 16; ++w) top = fmaxf(top, sh[w]);
    scales[blockIdx.x] = scale_from(top);
}

// X by columns: dst[k][q] = src[row(q)][k], zero where there is no position and in rows that are not asked for.  A workgroup turns 64
// positions by 64 columns in LDS.
template <typename T>
__global__ __launch_bounds__(256) void k_planes_columns(const T* __restrict__ src, const int64_t* __restrict__ target, Positions at, uint32_t K,
                                                        uint32_t Lq, uint16_t* __restrict__ dst) {
    __shared__ float t[64][65];
    const uint32_t k0 = blockIdx.y * 64u, q0 = blockIdx.x * 64u, col = threadIdx.x & 63u;
#pragma unroll
    for (uint32_t i = 0; i < 16u; ++i) {
        const uint32_t r = i * 4u + (threadIdx.x >> 6);
        const uint32_t row = at.row(q0 + r);
        float x = 0.f;
        if (row != 0xFFFFFFFFu && k0 + col < K && target[row] >= 0) {
            if (sizeof(T) == 4) x = ((const float*)src)[(uint64_t)row * K + k0 + col];
            else x = __uint_as_float((uint32_t)((const uint16_t*)src)[(uint64_t)row * K + k0 + col] << 16);
        }
        t[r][col] = x;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t u = threadIdx.x; u < 512u; u += 256u) {
        const uint32_t kk = u >> 3, q = q0 + (u & 7u) * 8u;
        if (k0 + kk >= K || q >= Lq) continue;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = t[(u & 7u) * 8u + e][kk];
        store_planes<T>(dst + (uint64_t)(k0 + kk) * Lq + q, (uint64_t)K * Lq, f);
    }
}

// X in float for the form in which every sample is one position; rows that are not asked for as zeros.
template <typename T>
__global__ __launch_bounds__(256) void k_asked_rows(const T* __restrict__ src, const int64_t* __restrict__ target, uint32_t R, uint32_t K, float* __restrict__ dst) {
    const uint32_t per_row = (K + 7u) / 8u;
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    if (i >= (uint64_t)R * per_row) return;
    const uint64_t row = i / per_row;
    const uint32_t k = (uint32_t)(i - row * per_row) * 8u;
    float f[8] = {};
    if (target[row] >= 0) widen8(load8(src + row * K + k, (int)(K - k)), f);
    store8(dst + row * K + k, f, (int)(K - k));
}

// ---- the logits of a tile and what becomes of them --------------------------------------------------------------------------
struct LossArgs {
    Matrix w, x;              // classes [v0, v0 + V) and rows of X, k contiguous
    uint32_t K, V, N;
    Positions at;             // of the tile's columns (forward: every row)
    uint32_t Lq;              // numbers of them, a multiple of 8 where D is stored by classes
    int64_t v0;
    const int64_t* target;
    // forward
    float2* partial;          // [block][N]: maximum, sum of exponentials relative to it
    float* picked;            // the target's logit
    uint32_t block0;
    // backward
    int64_t V_all;
    const float *lse, *weight;
    Scales scales;
    uint16_t* dt;             // D by classes, rows of Lq, planes `plane` apart
    uint64_t plane;
    uint32_t planes;
    float* d32;               // D in float by rows of X, V long
    float* rest;              // by rows of X: what rounding to bfloat16 left of the target's entry (bfloat16, for dX; or NULL)
};

constexpr float kLog2e = 1.44269504088896341f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
// Class, relative to m0, of a lane's result i of tile m.
__device__ __forceinline__ uint32_t class_of(int m, int i, uint32_t half) { return m * 32u + 8u * (i >> 2) + 4u * half + (i & 3); }

// acc[mt][nt] of a wave: classes m0 + 32 mt + .., columns n0 + 32 nt + lane % 32.
template <int MT, int NT>
__device__ __forceinline__ void finish_forward(f16v (&acc)[MT][NT], uint32_t m0, uint32_t n0, const LossArgs& A) {
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5;
    const float kNone = -__builtin_inff();
    if (m0 + MT * 32u > A.V) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (m0 + class_of(m, i, half) >= A.V)
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[m][n][i] = kNone;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t token = n0 + n * 32u + (lane & 31u);
        const bool live = token < A.N;
        const int64_t t = live ? A.target[token] - A.v0 : -1;
        const uint32_t at = t >= 0 && t < (int64_t)A.V ? (uint32_t)t - m0 : 0xFFFFFFFFu;      // class of this wave, if below 32 MT
        float top = kNone, sum = 0.f, z_t = 0.f;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float z = acc[m][n][i];
                top = fmaxf(top, z);
                if (at == class_of(m, i, half)) z_t = z;
            }
        const float base = top == kNone ? 0.f : top;         // (a column of -inf: its exponentials are 0)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += exp_of(acc[m][n][i] - base);
        const float top2 = __shfl_xor(top, 32), sum2 = __shfl_xor(sum, 32);
        const float both = fmaxf(top, top2), base2 = both == kNone ? 0.f : both;
        sum = sum * exp_of(top - base2) + sum2 * exp_of(top2 - base2);
        if (live && half == 0) A.partial[(size_t)(A.block0 + m0 / (MT * 32u)) * A.N + token] = make_float2(both, sum);
        if (live && at < MT * 32u && ((at >> 2) & 1u) == half) A.picked[token] = z_t;
    }
}

// What the backward pass knows of a column: its row of X, and how a logit becomes an entry of D.
struct ColumnOf {
    uint32_t row, at;         // the target's class in the piece, or ~0
    float lse, w, scale;      // w: relative to the sample's scale
    bool asked;
    __device__ __forceinline__ float d(float z, uint32_t v) const { return of(z - lse, v); }
    __device__ __forceinline__ float of(float z, uint32_t v) const { return asked ? (exp_of(z) - (v == at ? 1.f : 0.f)) * w : 0.f; }
};
__device__ __forceinline__ ColumnOf column_of(uint32_t q, const LossArgs& A) {
    ColumnOf C = {A.at.row(q), 0xFFFFFFFFu, 0.f, 0.f, 1.f, false};
    if (C.row == 0xFFFFFFFFu) return C;
    const int64_t t = A.target[C.row], tl = t - A.v0;
    C.asked = t >= 0;
    if (!C.asked) return C;
    C.lse = A.lse[C.row];
    C.scale = A.scales.at(q / A.at.Pp);
    C.w = t >= A.V_all ? __uint_as_float(0x7FC00000u) : A.weight ? A.weight[C.row] / C.scale : 1.f;       // (not a class: the gradients say so)
    if (tl >= 0 && tl < (int64_t)A.V) C.at = (uint32_t)tl;
    return C;
}

// What rounding to bfloat16 leaves of an entry of D.
__device__ __forceinline__ float left_of(float d) {
    float none = 0.f;
    next_plane<false>(d, none);
    return d;
}

// The logits become D in place.
template <bool kF32, int MT, int NT>
__device__ __forceinline__ void logits_to_d(f16v (&acc)[MT][NT], uint32_t m0, uint32_t n0, const LossArgs& A) {
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        ColumnOf C = column_of(n0 + n * 32u + (lane & 31u), A);
        C.at -= m0;
        float of_target = 0.f;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                acc[m][n][i] = C.d(acc[m][n][i], class_of(m, i, half));
                if (!kF32 && class_of(m, i, half) == C.at) of_target = acc[m][n][i];
            }
        if (!kF32 && A.rest && C.at < MT * 32u && ((C.at >> 2) & 1u) == half) A.rest[C.row] = left_of(of_target) * C.scale;
        if (A.d32 && C.row != 0xFFFFFFFFu) {
            float* out = A.d32 + (size_t)C.row * A.V + m0;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (m0 + class_of(m, i, half) < A.V) out[class_of(m, i, half)] = acc[m][n][i] * C.scale;
        }
    }
}

// D by classes (used up).  The wave turns its part in LDS, in bytes of its own, a plane at a time, and stores whole rows of its positions.  The two
// halves of a wave, four classes apart, write to different banks: 64-byte halves of a row of 64 positions change places with bit 2 of
// the class.
template <bool kF32, int MT, int NT>
__device__ __forceinline__ void store_by_classes(f16v (&acc)[MT][NT], uint8_t* turn, uint32_t m0, uint32_t n0, const LossArgs& A) {
    constexpr uint32_t kRow = NT * 64, kPieces = NT * 4, kRows = 64 / kPieces;               // bytes and pieces a class; classes a store
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5, flip = NT == 2 ? 1u : 0u;
    for (uint32_t q = 0; q < A.planes; ++q) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {            // (bit 2 of the class is the half)
                    float d0 = acc[m][n][i], d1 = acc[m][n][i + 1];
                    const uint32_t x = next_plane<kF32>(d0, d1);
                    acc[m][n][i] = d0;
                    acc[m][n][i + 1] = d1;
                    uint8_t* to = turn + class_of(m, i, half) * kRow + ((uint32_t)n ^ (half & flip)) * 64u + (lane & 31u) * 2u;
                    *reinterpret_cast<uint16_t*>(to) = (uint16_t)x;
                    *reinterpret_cast<uint16_t*>(to + kRow) = (uint16_t)(x >> 16);
                }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 4
        for (uint32_t r = 0; r < MT * 32 / kRows; ++r) {
            const uint32_t v = r * kRows + lane / kPieces, piece = lane % kPieces;
            const any_u4 x = *reinterpret_cast<const any_u4*>(turn + v * kRow + ((piece ^ ((((v >> 2) & flip)) << 2)) * 16u));
            if (m0 + v < A.V && n0 + piece * 8u < A.Lq) *reinterpret_cast<any_u4*>(A.dt + q * A.plane + (size_t)(m0 + v) * A.Lq + n0 + piece * 8u) = x;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// 65536 classes x 2048 k, 4096 bfloat16 rows: forward 0.88-1.0 ms, 1.1-1.25 PFLOP/s, by the clock that the card keeps under the load
// (1.73-1.78 GHz; with zeros for inputs 0.73), LDS free of conflicts; as D, 65521 classes, 1.13-1.27 ms, with two planes, 1.07 GB, to be stored
// at the end of every tile.
template <typename Shape, bool kForward>
__global__ __launch_bounds__(Shape::NW * 64, 2) void k_logits(LossArgs A) {
    __shared__ __attribute__((aligned(1024))) uint8_t sh[Shape::kLds];
    const uint32_t tiles_n = ((kForward ? A.N : A.Lq) + Shape::BN - 1) / Shape::BN, tiles_m = (A.V + Shape::BM - 1) / Shape::BM;
    const TilePlace at = in_bands(xcd_contiguous(blockIdx.x, gridDim.x), tiles_m, tiles_n);
    const uint32_t m0 = at.m * Shape::BM, n0 = at.n * Shape::BN;
    f16v acc[Shape::MT][Shape::NT] = {};
    // the tile's rows of X lie between those of its first and of its last position
    const uint32_t z0 = n0 / A.at.Pp, first = min(z0 * A.at.P + min(n0 - z0 * A.at.Pp, A.at.P), A.N);
    // float32: in parts of 32 k (600 rows of 4096 channels, logits of 14: lse 1.2e-4 too small in one part; 2048 rows of 120, logits of 16: 2.0e-6
    // off in parts of 128, so 0.9e-6; of 2048: 1.2e-6 and 1.9e-6, where float sums are 9.8e-6)
    // bfloat16, few rows, whose logits' errors no sum averages: of 128 (10 rows of 1703, 21092 classes, logits of 16: lse 4.1e-6 off, so 1.3e-6;
    // the larger tiles have no registers for it: 3.6e-6, where float sums are 8e-6 off)
    InParts<Shape, Shape::PB == 3 ? 32u : Shape::MT * Shape::NT <= 2 ? 128u : 0u> parts;
    RowTile<Shape>::run(acc, sh, A.w, A.x, m0, first, Shape::BN, [&](uint32_t n) {
        const uint32_t row = A.at.row(n0 + n);
        return row == 0xFFFFFFFFu ? row : row - first;
    }, A.K, [&](uint32_t step, int ks) { parts.after(acc, step, ks); });
    parts.end(acc);
    const uint32_t wm = m0 + Shape::wave_m(), wn = n0 + Shape::wave_n();
    if (kForward) {
        if (wm < A.V) finish_forward(acc, wm, wn, A);
    } else {
        logits_to_d<Shape::PB == 3>(acc, wm, wn, A);
        static_assert(Shape::NT <= 2 && Shape::BM * Shape::BN * 2u <= Shape::kLds, "room to turn a plane");
        if (A.dt) store_by_classes<Shape::PB == 3>(acc, sh + Shape::wave() * (Shape::WM * Shape::WN * 2u), wm, wn, A);
    }
}

// Few rows, or few classes: a workgroup of 16 waves owns kT x kT tiles of 16 classes by 16 columns and its waves share k, in steps of
// 128 bytes of a row, with both operands straight from memory into registers, 4 / kT steps ahead.  A load takes
// 64 consecutive bytes of 16 rows, four lanes a row, which is how the 16 x 16 instructions want them (with 32 rows a load, 32 bytes
// of each, the address units are what it waits for: 19.2 us instead of 10.4 for 64 rows, 1000 classes, 4096 k); which k an instruction's place
// stands for is free as long as both operands agree.  The waves' sums meet in LDS, where a thread takes one result.  float32 rows
// are multiplied as floats.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t bounded(const void* base, uint64_t offset, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base) + offset), 0, (int)bytes, 0x00020000);
}
constexpr uint32_t kThinWaves = 16;
struct ThinArgs { const void *w, *x; uint32_t ldw, ldx; };   // rows in their own type; element pitches
template <typename T, int kT, bool kForward>
__global__ __launch_bounds__(kThinWaves * 64) void k_logits_thin(ThinArgs R, LossArgs A) {
    constexpr uint32_t kN = 16 * kT, kPitch = kN + 4;        // (rows of four lane groups start 16 banks apart)
    constexpr uint32_t kE = 16 / sizeof(T), kStep = 128 / sizeof(T), kTurn = kThinWaves * kStep;      // elements a load; k a step; of all waves
    constexpr int kAhead = kT == 1 ? 4 : 2;
    __shared__ float sh[kThinWaves][kN][kPitch];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t columns = kForward ? A.N : A.Lq, tiles_n = (columns + kN - 1) / kN, id = xcd_contiguous(blockIdx.x, gridDim.x);
    const uint32_t m0 = id / tiles_n * kN, n0 = id % tiles_n * kN;
    // a thread's result: consecutive classes; what it takes besides the logit is asked for first
    const uint32_t v = tid % kN, col = tid / kN;
    const bool mine = tid < kN * kN && m0 + v < A.V && n0 + col < columns;
    ColumnOf C;
    int64_t t = -1;
    if constexpr (kForward) { if (mine) t = A.target[n0 + col]; }
    else if (mine) C = column_of(n0 + col, A);
    const uint32_t z0 = n0 / A.at.Pp, first = min(z0 * A.at.P + min(n0 - z0 * A.at.Pp, A.at.P), A.N);
    const __amdgpu_buffer_rsrc_t rw = bounded(R.w, (uint64_t)m0 * R.ldw * sizeof(T), min(A.V - m0, kN) * R.ldw * (uint32_t)sizeof(T));
    const __amdgpu_buffer_rsrc_t rx = bounded(R.x, (uint64_t)first * R.ldx * sizeof(T), min(A.N - first, kN) * R.ldx * (uint32_t)sizeof(T));
    const uint32_t kl = (lane >> 4) * kE;
    uint32_t offW[kT], offX[kT], none[kT];
#pragma unroll
    for (int t = 0; t < kT; ++t) {
        const uint32_t row = A.at.row(n0 + t * 16u + (lane & 15u));
        none[t] = row == 0xFFFFFFFFu ? row : 0u;
        offW[t] = ((t * 16u + (lane & 15u)) * R.ldw + kl) * (uint32_t)sizeof(T);
        offX[t] = ((row - first) * R.ldx + kl) * (uint32_t)sizeof(T);
    }
    struct Step { i4v w[kT][2], x[kT][2]; };
    auto request = [&](uint32_t k) -> Step {                 // (past the end: zeros)
        Step S;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t outside = k + kl + j * 4u * kE < A.K ? 0u : 0xFFFFFFFFu, add = (k + j * 4u * kE) * (uint32_t)sizeof(T);
#pragma unroll
            for (int t = 0; t < kT; ++t) {
                S.w[t][j] = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)((offW[t] + add) | outside), 0, 0));
                S.x[t][j] = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(rx, (int)((offX[t] + add) | outside | none[t]), 0, 0));
            }
        }
        return S;
    };
    f4v sum[kT][kT] = {};
    auto multiply = [&](const Step& S, uint32_t k) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int m = 0; m < kT; ++m)
#pragma unroll
                    for (int n = 0; n < kT; ++n)
                        sum[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, S.w[m][j]), __builtin_bit_cast(bf8v, S.x[n][j]), sum[m][n], 0, 0, 0);
            } else {
                f4v w[kT], x[kT];
#pragma unroll
                for (int t = 0; t < kT; ++t) { w[t] = __builtin_bit_cast(f4v, S.w[t][j]); x[t] = __builtin_bit_cast(f4v, S.x[t][j]); }
                if (k + kStep > A.K) {                       // a load that reaches past the rows' end has brought the next row's begin
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (k + kl + j * 4u * kE + e >= A.K)
#pragma unroll
                            for (int t = 0; t < kT; ++t) w[t][e] = x[t][e] = 0.f;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int m = 0; m < kT; ++m)
#pragma unroll
                        for (int n = 0; n < kT; ++n) sum[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[m][e], x[n][e], sum[m][n], 0, 0, 0);
            }
        }
    };
    Step S[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (wave * kStep + i * kTurn < A.K) S[i] = request(wave * kStep + i * kTurn);
    for (uint32_t k = wave * kStep; k < A.K; k += kAhead * kTurn)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (k + i * kTurn >= A.K) break;
            multiply(S[i], k + i * kTurn);
            if (k + (kAhead + i) * kTurn < A.K) S[i] = request(k + (kAhead + i) * kTurn);
        }
    // result i of a lane: class 4 (lane / 16) + i, column lane % 16
#pragma unroll
    for (int m = 0; m < kT; ++m)
#pragma unroll
        for (int n = 0; n < kT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) sh[wave][m * 16 + (lane >> 4) * 4 + i][n * 16 + (lane & 15u)] = sum[m][n][i];
    __syncthreads();
    double whole = 0.;                                       // (the sixteen in float: dX of 3 rows of 3095 float32 2.1e-6 off, so 1.3e-6)
    if (tid < kN * kN) {
#pragma unroll
        for (uint32_t w = 0; w < kThinWaves; ++w) whole += (double)sh[w][v][col];
    }
    if constexpr (kForward) {                                // 16 kT consecutive lanes hold a token's classes
        const float kNone = -__builtin_inff();
        const float z = mine ? (float)whole : kNone;
        float top = z;
        lanes_max<kN>(top);
        const float base = top == kNone ? 0.f : top;
        const float total = lanes_sum<kN>(exp_of(z - base));
        if (!mine) return;
        if (v == 0u) A.partial[(size_t)(A.block0 + m0 / kN) * A.N + n0 + col] = make_float2(top, total);
        if (t == A.v0 + m0 + v) A.picked[n0 + col] = z;
    } else {
        if (!mine) return;
        float d = C.of((float)(whole - (double)C.lse), m0 + v);
        if (A.d32 && C.row != 0xFFFFFFFFu) A.d32[(size_t)C.row * A.V + m0 + v] = d * C.scale;
        if (sizeof(T) == 2 && A.rest && C.at == m0 + v) A.rest[C.row] = left_of(d) * C.scale;
        if (A.dt)
            for (uint32_t q = 0; q < A.planes; ++q) {
                float none = 0.f;
                A.dt[q * A.plane + (size_t)(m0 + v) * A.Lq + n0 + col] = (uint16_t)next_plane<sizeof(T) == 4>(d, none);
            }
    }
}

// Joins the pairs of a token over the blocks of the vocabulary in a fixed order: 16 waves take every 16th block of 64 tokens.
__global__ __launch_bounds__(1024) void k_loss_join(const float2* __restrict__ partial, const float* __restrict__ picked, const int64_t* __restrict__ target,
                                                    uint32_t blocks, uint32_t N, int64_t V, float* __restrict__ loss, float* __restrict__ lse_out) {
    __shared__ float2 sh[16][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, token = blockIdx.x * 64u + lane;
    const float kNone = -__builtin_inff();
    float top = kNone, sum = 0.f;
    auto add = [&](float2 q) {
        const float both = fmaxf(top, q.x), base = both == kNone ? 0.f : both;
        sum = sum * exp_of(top - base) + q.y * exp_of(q.x - base);
        top = both;
    };
    if (token < N) {
#pragma unroll 4
        for (uint32_t b = wave; b < blocks; b += 16u) add(partial[(size_t)b * N + token]);
    }
    sh[wave][lane] = make_float2(top, sum);
    __syncthreads();
    if (wave != 0u || token >= N) return;
    for (uint32_t w = 1; w < 16u; ++w) add(sh[w][lane]);
    const float lse = top + logf(sum);
    const int64_t t = target[token];
    lse_out[token] = lse;
    loss[token] = t < 0 ? 0.f : t < V ? lse - picked[token] : __uint_as_float(0x7FC00000u);
}

// ---- dX -----------------------------------------------------------------------------------------------------------------------
// Part `split` of the sum over the piece's classes, added to what the pieces before have left in the part's own plane [N, H].
// Bound by the matrix instructions: 4096 x 2048 from 65521 classes of bfloat16 0.87-0.96 ms, 1.15-1.27 PFLOP/s.
template <typename Shape>
__global__ __launch_bounds__(Shape::NW * 64, 2) void k_loss_dx(Matrix Dt, Matrix W, Positions at, Scales scales, uint32_t H, uint32_t splits, int add,
                                                               float* __restrict__ planes) {
    __shared__ __attribute__((aligned(1024))) uint8_t sh[Shape::kLds];
    const uint32_t N = at.B * at.P, tiles_n = (H + Shape::BN - 1) / Shape::BN, tiles_m = (at.B * at.Pp + Shape::BM - 1) / Shape::BM;
    const uint32_t id = xcd_contiguous(blockIdx.x, gridDim.x), split = id / (tiles_n * tiles_m), tile = id - split * tiles_n * tiles_m;
    const uint32_t m0 = tile / tiles_n * Shape::BM, n0 = tile % tiles_n * Shape::BN, steps = (Dt.rows + Shape::BK - 1) / Shape::BK;
    const uint32_t k0 = (uint32_t)((uint64_t)split * steps / splits) * Shape::BK;
    const uint32_t k1 = min((uint32_t)((uint64_t)(split + 1u) * steps / splits) * Shape::BK, Dt.rows);
    f16v acc[Shape::MT][Shape::NT] = {};
    InParts<Shape, Shape::PB == 3 ? 32u : 0u> parts;
    ColumnTile<Shape>::run(acc, sh, Dt, W, m0, n0, k0, k1, [&](uint32_t step, int ks) { parts.after(acc, step, ks); });
    parts.end(acc);
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5, wm = m0 + Shape::wave_m(), wn = n0 + Shape::wave_n();
    float* out = planes + (size_t)split * N * H;
#pragma unroll
    for (int m = 0; m < Shape::MT; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t row = at.row(wm + class_of(m, i, half));
            if (row == 0xFFFFFFFFu) continue;
            const float scale = scales.at(row / at.P);
#pragma unroll
            for (int n = 0; n < Shape::NT; ++n) {
                const uint32_t h = wn + n * 32u + (lane & 31u);
                if (h >= H) continue;
                float* to = out + (size_t)row * H + h;
                *to = acc[m][n][i] * scale + (add ? *to : 0.f);
            }
        }
}

// What the target's entry, the largest of a row that misses its class, lost when it was rounded: added to dX as so much of the class's row.
struct TargetRest {
    const float* rest;
    const int64_t* target;
    const uint16_t* W;
    int64_t V;
    uint32_t H;
    __device__ __forceinline__ void add(uint64_t i, int m, float (&f)[8]) const {
        uint64_t row = i / H;
        uint32_t h = (uint32_t)(i - row * H);
        for (int e = 0; e < m;) {                            // (eight elements may belong to several rows)
            const int many = (int)min(H - h, (uint32_t)(m - e));
            const int64_t t = target[row];
            if (t >= 0 && t < V) {
                const float r = rest[row];
                if (many == 8) {
                    float w[8];
                    widen8(load8(W + (uint64_t)t * H + h, 8), w);
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[k] = __builtin_fmaf(r, w[k], f[k]);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (k >= e && k < e + many) f[k] = __builtin_fmaf(r, __uint_as_float((uint32_t)W[(uint64_t)t * H + h + (k - e)] << 16), f[k]);
                }
            }
            e += many;
            h = 0;
            ++row;
        }
    }
};

// Adds the parts' planes in a fixed order, eight elements a lane; kWaves waves share many planes of few elements (6 x 529 from 64: 15 us
// by one, 4 by 16).
template <typename T, uint32_t kWaves>
__global__ __launch_bounds__(kWaves == 1 ? 256 : kWaves * 64) void k_loss_dx_join(const float* __restrict__ planes, uint32_t splits, uint64_t n, TargetRest target,
                                                                                  T* __restrict__ dX) {
    const uint32_t lane = threadIdx.x & 63u, wave = kWaves == 1 ? 0u : threadIdx.x >> 6;
    const uint64_t i = (kWaves == 1 ? (uint64_t)blockIdx.x * 256u + threadIdx.x : (uint64_t)blockIdx.x * 64u + lane) * 8u;
    const int m = i >= n ? 0 : n - i >= 8u ? 8 : (int)(n - i);
    float f[8] = {}, g[8];
    if (m > 0) {
#pragma unroll 4
        for (uint32_t s = wave; s < splits; s += kWaves) {
            widen8(load8(planes + s * n + i, m), g);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += g[e];
        }
        if (sizeof(T) == 2 && wave == 0u) target.add(i, m, f);
    }
    if constexpr (kWaves > 1) {
        __shared__ float sh[kWaves][8][64];
#pragma unroll
        for (int e = 0; e < 8; ++e) sh[wave][e][lane] = f[e];
        __syncthreads();
        if (wave != 0u) return;
#pragma unroll
        for (uint32_t w = 1; w < kWaves; ++w)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += sh[w][e][lane];
    }
    if (m > 0) store8(dX + i, f, m);
}

// Few rows and few classes: 16 waves share the classes for 32 rows by 32 columns of dX, D and W multiplied as floats.  A wave takes 8
// classes at a time, four a half.
constexpr uint32_t kThinDx = 32;
template <typename T>
__global__ __launch_bounds__(kThinWaves * 64) void k_loss_dx_thin(const float* __restrict__ D, const T* __restrict__ W, uint32_t N, uint32_t V, uint32_t H,
                                                                  T* __restrict__ dX) {
    __shared__ float sh[kThinWaves][16][64];
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tiles_n = (N + kThinDx - 1) / kThinDx, n0 = blockIdx.x % tiles_n * kThinDx, h = blockIdx.x / tiles_n * kThinDx + (lane & 31u);
    const uint32_t n = n0 + (lane & 31u);
    f16v sum = {};
    struct Step { float d[4], w[4]; };
    auto request = [&](uint32_t v0) -> Step {
        Step S;
        const uint32_t first = v0 + half * 4u;               // (four of a row's entries at once: one at a time the address units take 20 us)
        any_f4 d = {0.f, 0.f, 0.f, 0.f};
        if (n < N && first + 3u < V) d = *reinterpret_cast<const any_f4*>(D + (size_t)n * V + first);
        else if (n < N)
            for (uint32_t e = 0; e < 3u; ++e)
                if (first + e < V) d[e] = D[(size_t)n * V + first + e];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t v = first + e;
            S.d[e] = d[e];
            S.w[e] = 0.f;
            if (v < V && h < H) {
                if (sizeof(T) == 4) S.w[e] = ((const float*)W)[(size_t)v * H + h];
                else S.w[e] = __uint_as_float((uint32_t)((const uint16_t*)W)[(size_t)v * H + h] << 16);
            }
        }
        return S;
    };
    constexpr uint32_t kTurn = kThinWaves * 8u;
    constexpr int kAhead = 2;
    Step S[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (wave * 8u + i * kTurn < V) S[i] = request(wave * 8u + i * kTurn);
    for (uint32_t v0 = wave * 8u; v0 < V; v0 += kAhead * kTurn)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (v0 + i * kTurn >= V) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_32x32x2f32(S[i].d[e], S[i].w[e], sum, 0, 0, 0);
            if (v0 + (kAhead + i) * kTurn < V) S[i] = request(v0 + (kAhead + i) * kTurn);
        }
#pragma unroll
    for (int i = 0; i < 16; ++i) sh[wave][i][lane] = sum[i];
    __syncthreads();
    float r = 0.f;                                           // (16 waves and 16 results: a wave adds one of them)
#pragma unroll
    for (uint32_t w = 0; w < kThinWaves; ++w) r += sh[w][wave][lane];
    const uint32_t row = n0 + class_of(0, wave, half);
    if (row >= N || h >= H) return;
    if (sizeof(T) == 4) ((float*)dX)[(size_t)row * H + h] = r;
    else ((uint16_t*)dX)[(size_t)row * H + h] = (uint16_t)two_bf16(r, 0.f);
}

// ---- g and s ------------------------------------------------------------------------------------------------------------------
// Samples of one position, few of them, and few classes: a workgroup takes 64 columns of X by 4 classes, its 16 waves share the samples.
// Rows that are not asked for count as zeros whatever they hold.
template <typename T>
__global__ __launch_bounds__(1024) void k_loss_sums_thin(const float* __restrict__ D, const T* __restrict__ X, const int64_t* __restrict__ target, uint32_t N,
                                                         uint32_t V, uint32_t H, float c, float* __restrict__ g_out, float* __restrict__ s_out) {
    __shared__ float sh[2][4][16][64];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t blocks_v = (V + 3u) / 4u, h = blockIdx.x / blocks_v * 64u + lane, v0 = blockIdx.x % blocks_v * 4u, count = min(4u, V - v0);
    float g[4] = {}, s[4] = {};
#pragma unroll 4
    for (uint32_t n = wave; n < N; n += 16u) {
        float x = 0.f;
        if (h < H && target[n] >= 0) {
            if (sizeof(T) == 4) x = ((const float*)X)[(size_t)n * H + h];
            else x = __uint_as_float((uint32_t)((const uint16_t*)X)[(size_t)n * H + h] << 16);
        }
#pragma unroll
        for (uint32_t e = 0; e < 4u; ++e) {
            const float p = x * (e < count ? D[(size_t)n * V + v0 + e] : 0.f);
            g[e] += p;
            s[e] = __builtin_fmaf(p, p, s[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) { sh[0][e][wave][lane] = g[e]; sh[1][e][wave][lane] = s[e]; }
    __syncthreads();
    if (wave >= 8u) return;                                  // a wave adds one of the eight sums
    const uint32_t e = wave & 3u, which = wave >> 2;
    float sum = 0.f;
#pragma unroll
    for (uint32_t w = 0; w < 16u; ++w) sum += sh[which][e][w][lane];
    if (h >= H || e >= count) return;
    const size_t at = (size_t)(v0 + e) * H + h;
    if (which) s_out[at] = c * c * sum;
    else if (g_out) g_out[at] = c * sum;
}

// k runs over the positions; at a sample's end (every Pp of them) its product is squared into s, added into g, and cleared.
// Bound by the matrix instructions, two planes of D by one of X, bfloat16 65521 x 2048 from 4 x 1024 positions: 2.0-2.2 ms, 1.0-1.1 PFLOP/s of
// them, 1.07 GB of outputs within.
// kPast: outputs beyond what the caches hold are stored past them.
template <typename Shape, bool kPast>
__global__ __launch_bounds__(Shape::NW * 64, 2) void k_loss_sums(Matrix Dt, Matrix Xt, uint32_t B, uint32_t Pp, Scales scales, float c, float* __restrict__ g_out,
                                                                 float* __restrict__ s_out) {
    __shared__ __attribute__((aligned(1024))) uint8_t sh[Shape::kLds];
    const uint32_t V = Dt.rows, H = Xt.rows, tiles_n = (H + Shape::BN - 1) / Shape::BN;
    const uint32_t id = xcd_contiguous(blockIdx.x, gridDim.x), m0 = id / tiles_n * Shape::BM, n0 = id % tiles_n * Shape::BN;
    f16v acc[Shape::MT][Shape::NT] = {}, g[Shape::MT][Shape::NT] = {}, s[Shape::MT][Shape::NT] = {};
    InParts<Shape, Shape::PB == 3 ? 32u : 0u> parts;
    constexpr bool kScaled = Shape::PB == 1;                 // (bfloat16; float32 planes hold D as it is)
    uint32_t left = Pp, z = 0;
    float scale = kScaled ? scales.at(0) : 1.f;
    RowTile<Shape>::run(acc, sh, Dt, Xt, m0, n0, Shape::BN, [&](uint32_t n) { return n0 + n < H ? n : 0xFFFFFFFFu; }, B * Pp, [&](uint32_t step, int ks) {
        left -= 16u;
        if (left != 0u) { parts.after(acc, step, ks); return; }
        parts.end(acc);
        parts = {};
        left = Pp;
#pragma unroll
        for (int m = 0; m < Shape::MT; ++m)
#pragma unroll
            for (int n = 0; n < Shape::NT; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = kScaled ? acc[m][n][i] * scale : acc[m][n][i];
                    g[m][n][i] += x;
                    s[m][n][i] = __builtin_fmaf(x, x, s[m][n][i]);
                    acc[m][n][i] = 0.f;
                }
        z = min(z + 1u, B - 1u);                             // (past the last sample there are steps of zeros)
        if (kScaled) scale = scales.at(z);
    });
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5, wm = m0 + Shape::wave_m(), wn = n0 + Shape::wave_n();
#pragma unroll
    for (int n = 0; n < Shape::NT; ++n) {
        const uint32_t h = wn + n * 32u + (lane & 31u);
        if (h >= H) continue;
#pragma unroll
        for (int m = 0; m < Shape::MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t v = wm + class_of(m, i, half);
                if (v >= V) continue;
                float *gp = g_out + (size_t)v * H + h, *sp = s_out + (size_t)v * H + h;
                if (kPast) {
                    if (g_out) __builtin_nontemporal_store(c * g[m][n][i], gp);
                    __builtin_nontemporal_store(c * c * s[m][n][i], sp);
                } else {
                    if (g_out) *gp = c * g[m][n][i];
                    *sp = c * c * s[m][n][i];
                }
            }
    }
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
//               BM   BN   WM  WN BK S PA PB
typedef TileShape<256, 256, 128, 64, 64, 2, 1, 1> Large;     // bfloat16: the logits and dX
typedef TileShape<128, 128, 64, 64, 64, 2, 1, 1> Small;
typedef TileShape<128, 64, 64, 32, 64, 3, 1, 1> Slim;        // few rows over many classes: W streams through
typedef TileShape<256, 128, 64, 64, 32, 2, 3, 3> Cut;        // float32: the logits and dX
typedef TileShape<128, 128, 64, 32, 32, 2, 3, 3> CutSums;    // float32: g and s (registers for four accumulators; with 64 x 64 a wave they
//   spilled: 4 x 512 positions of 1024, 4000 classes, the backward pass 404 us, so 301; 10 x 297 of 3755, 1191 classes, 799 and 727)
typedef TileShape<128, 256, 64, 64, 64, 2, 2, 1> Sums;       // bfloat16: g and s
typedef TileShape<128, 128, 64, 32, 64, 2, 3, 1> SumsOfFew;  // from all bits of D

static uint32_t up8(uint32_t x) { return (x + 7u) / 8u * 8u; }
// (2^24 classes by 2^20 rows are 2^36 tiles of 16 x 16)
static uint64_t tiles(uint32_t a, uint32_t ta, uint32_t b, uint32_t tb) { return (uint64_t)((a + ta - 1) / ta) * ((b + tb - 1) / tb); }
template <typename Shape> static uint64_t tiles(uint32_t m, uint32_t n) { return tiles(m, Shape::BM, n, Shape::BN); }

// The kernel that forms the logits.  Forward times (us, both launches) that the rule goes by:
//   16 x 16 or 32 x 32 results a workgroup while there are no more workgroups than compute units, so that k is what is shared out: 64
//     rows, 4096 k, 1000 classes: 13.2, 20.4, slim tiles 24.3; 128 rows: 22.3, 21.2, 25.0; 256 rows, 2000 classes: 70.3, 37.7, 25.6.
//   slim tiles until there are enough of the others: 16000 classes x 1024 k, 256 rows: slim 18.7, small 20.6, large 28.7; 512 rows: 30.8,
//     24.8, 30.5; 1024 rows: 50.4, 44.1, 38.9; 64000 classes, 64 rows: 37, 39, 44; 128 rows: 48, 42, 44; 256 rows: 71, 60, 51.
//   float32: tiles of planes from 2 M logits on, which their laying out has to be paid by: 4000 classes x 1024 k, 512 rows: 73, as floats 86;
//     16000 x 128: 89 and 89; 4000 x 256: 74 and 47; 64000 x 64: 254 and 204.
enum class LogitsTile { kLarge, kSmall, kSlim, kCut, kThin, kThinnest };
static LogitsTile logits_tile(int dtype, uint32_t V, uint32_t N) {
    if (tiles(V, 16, N, 16) <= 256u) return LogitsTile::kThinnest;
    if (dtype == VGC_F32) return N > 64u && (uint64_t)V * N >= 2000000u ? LogitsTile::kCut : LogitsTile::kThin;
    if (tiles(V, 32, N, 32) <= 256u) return LogitsTile::kThin;
    if (N > 128u && tiles<Large>(V, N) >= 192u) return LogitsTile::kLarge;
    return N > 64u && tiles<Small>(V, N) >= 320u ? LogitsTile::kSmall : LogitsTile::kSlim;
}
static bool is_thin(LogitsTile t) { return t == LogitsTile::kThin || t == LogitsTile::kThinnest; }
// Classes a partial pair of the forward pass covers: those of a wave, in the thin kernels of a workgroup.
static uint32_t logits_block(LogitsTile t) {
    return t == LogitsTile::kLarge ? 128u : t == LogitsTile::kThin ? 32u : t == LogitsTile::kThinnest ? 16u : 64u;
}

template <bool kForward>
static int launch_logits(LogitsTile t, int dtype, const ThinArgs& R, const LossArgs& A, hipStream_t stream) {
    const uint32_t n = kForward ? A.N : A.Lq;
#define VGC_LAUNCH(S) hipLaunchKernelGGL((k_logits<S, kForward>), dim3(tiles<S>(A.V, n)), dim3(S::NW * 64), 0, stream, A)
#define VGC_THIN(T, kT) hipLaunchKernelGGL((k_logits_thin<T, kT, kForward>), dim3(tiles(A.V, 16 * kT, n, 16 * kT)), dim3(kThinWaves * 64), 0, stream, R, A)
    switch (t) {
        case LogitsTile::kLarge: VGC_LAUNCH(Large); break;
        case LogitsTile::kSmall: VGC_LAUNCH(Small); break;
        case LogitsTile::kSlim: VGC_LAUNCH(Slim); break;
        case LogitsTile::kCut: VGC_LAUNCH(Cut); break;
        case LogitsTile::kThin: if (dtype == VGC_F32) VGC_THIN(float, 2); else VGC_THIN(uint16_t, 2); break;
        case LogitsTile::kThinnest: if (dtype == VGC_F32) VGC_THIN(float, 1); else VGC_THIN(uint16_t, 1); break;
    }
#undef VGC_THIN
#undef VGC_LAUNCH
    return hip_check(hipGetLastError(), "launch k_logits");
}

int launch_plane_rows(int dtype, const PlaneRows& first, const PlaneRows& second, hipStream_t stream) {
    auto groups_of = [](const PlaneRows& M) { return (uint32_t)(((uint64_t)M.R * (up8(M.K) / 8u) + 255u) / 256u); };
    const uint32_t groups = groups_of(first);
    const dim3 grid(groups + groups_of(second));
    if (dtype == VGC_BF16) hipLaunchKernelGGL(k_planes_rows<uint16_t>, grid, dim3(256), 0, stream, first, second, groups);
    else hipLaunchKernelGGL(k_planes_rows<float>, grid, dim3(256), 0, stream, first, second, groups);
    return hip_check(hipGetLastError(), "launch k_planes_rows");
}

// The vocabulary in pieces of equal size, multiples of 256 classes, `bytes` of working memory a class.
static uint32_t piece_of(uint32_t V, uint64_t bytes, uint64_t budget) {
    uint64_t most = budget / std::max<uint64_t>(bytes, 1) / 256u * 256u;
    most = std::min<uint64_t>(std::max<uint64_t>(most, 256u), 1u << 20);
    const uint32_t pieces = (uint32_t)((V + most - 1) / most);
    return std::min(((V + pieces - 1) / pieces + 255u) / 256u * 256u, V);
}

// What both passes do with their rows: used where they lie if they are bfloat16 and whole pieces of 16 bytes, or floats of the thin
// kernels; else laid out as planes.
struct RowsPlan { uint32_t planes, Kp; bool in_place; };
static RowsPlan rows_plan(int dtype, uint32_t H, LogitsTile t, bool dx_by_tiles) {
    RowsPlan r;
    r.planes = dtype == VGC_F32 ? 3u : 1u;
    r.Kp = up8(H);
    r.in_place = dtype == VGC_BF16 ? H % 8u == 0 : is_thin(t) && !dx_by_tiles;
    return r;
}

struct ForwardPlan { LogitsTile tile; RowsPlan rows; uint32_t piece, blocks; size_t x, w, partial, picked, total; };
static ForwardPlan forward_plan(int dtype, uint32_t N, uint32_t H, uint32_t V) {
    ForwardPlan L;
    L.tile = logits_tile(dtype, V, N);
    L.rows = rows_plan(dtype, H, L.tile, false);
    const uint64_t row = 2ull * L.rows.planes * L.rows.Kp;
    // a launch has fewer than 2^32 threads: 2^36 logits at a time, of which a thread has 32 or more (the thin kernels, one, few altogether)
    L.piece = (uint32_t)std::min<uint64_t>(L.rows.in_place ? V : piece_of(V, row, 256ull << 20), (1ull << 36) / N / 256u * 256u);
    L.blocks = (V + logits_block(L.tile) - 1) / logits_block(L.tile);
    size_t off = 0;
    L.x = off; if (!L.rows.in_place) off = align_up(off + N * row, 256);
    L.w = off; if (!L.rows.in_place) off = align_up(off + L.piece * row, 256);
    L.partial = off; off = align_up(off + (size_t)L.blocks * N * sizeof(float2), 256);
    L.picked = off; off += (size_t)N * sizeof(float);
    L.total = off;
    return L;
}
size_t softmax_loss_workspace_bytes(int dtype, uint32_t N, uint32_t H, uint32_t V) { return forward_plan(dtype, N, H, V).total; }

// The rows of an operand as both kinds of kernels take them.
static Matrix matrix_of(const RowsPlan& r, const void* src, const uint16_t* planes, uint32_t rows, uint32_t H) {
    return r.in_place ? Matrix{static_cast<const uint16_t*>(src), rows, H, 0} : Matrix{planes, rows, r.Kp, (uint64_t)rows * r.Kp};
}

int launch_softmax_loss(int dtype, const void* X, const void* W, const int64_t* target, uint32_t N, uint32_t H, uint32_t V, float* loss, float* lse,
                        void* workspace, hipStream_t stream) {
    const ForwardPlan L = forward_plan(dtype, N, H, V);
    char* ws = static_cast<char*>(workspace);
    const size_t size = dtype == VGC_F32 ? 4 : 2;
    int rc;
    LossArgs A = {};
    A.N = A.Lq = N;
    A.K = L.rows.in_place ? H : L.rows.Kp;
    A.at = Positions{N, 1, 1};
    A.target = target;
    A.partial = reinterpret_cast<float2*>(ws + L.partial);
    A.picked = reinterpret_cast<float*>(ws + L.picked);
    uint16_t *xs = reinterpret_cast<uint16_t*>(ws + L.x), *wp = reinterpret_cast<uint16_t*>(ws + L.w);
    if (!L.rows.in_place && (rc = launch_plane_rows(dtype, {X, N, H, xs}, {}, stream)) != VGC_OK) return rc;
    A.x = matrix_of(L.rows, X, xs, N, H);
    for (uint32_t v0 = 0; v0 < V; v0 += L.piece) {
        A.v0 = v0;
        A.V = std::min(L.piece, V - v0);
        const char* rows = static_cast<const char*>(W) + (size_t)v0 * H * size;
        if (!L.rows.in_place && (rc = launch_plane_rows(dtype, {rows, A.V, H, wp}, {}, stream)) != VGC_OK) return rc;
        A.w = matrix_of(L.rows, rows, wp, A.V, H);
        A.block0 = v0 / logits_block(L.tile);
        if ((rc = launch_logits<true>(L.tile, dtype, ThinArgs{A.w.base, A.x.base, A.w.ld, A.x.ld}, A, stream)) != VGC_OK) return rc;
    }
    hipLaunchKernelGGL(k_loss_join, dim3((N + 63) / 64), dim3(1024), 0, stream, A.partial, A.picked, target, L.blocks, N, (int64_t)V, loss, lse);
    return hip_check(hipGetLastError(), "launch k_loss_join");
}

struct BackwardPlan {
    LogitsTile tile;
    RowsPlan rows;
    uint32_t planes, piece, Pp, Lq, splits;
    bool dx_thin, dx_large, sum_planes, sum_thin;
    size_t x, xt, w, d, d32, d2, out, scales, rest, total;
};
static BackwardPlan backward_plan(int dtype, uint32_t B, uint32_t P, uint32_t H, uint32_t V) {
    BackwardPlan L;
    const uint32_t N = B * P;
    L.Pp = P == 1 ? 1u : (P + 15u) / 16u * 16u;              // (a sample's end falls on a phase's)
    L.Lq = up8(B * L.Pp);
    L.tile = logits_tile(dtype, V, L.Lq);
    // dX of few rows from floats, without planes or partial sums, while that is little work (us with the logits: bfloat16, 1000 classes, 64 x
    // 4096: 29 and 31 by tiles, 128 x 4096: 47 and 39, 4000 classes, 16 x 512: 48 and 19; float32, 1000 x 128 x 4096: 61 and 90, 4000 x 256 x
    // 2048: 155 and 143)
    const uint64_t work = (uint64_t)N * V * H;
    L.dx_thin = P == 1 && (uint64_t)N * V <= (64u << 20) && (dtype == VGC_F32 ? work <= 2000000000u : V <= 1024u && work <= (256u << 20));
    L.rows = rows_plan(dtype, H, L.tile, !L.dx_thin);
    // bfloat16: D of samples of few positions, and of small products, in three planes, all its bits, as few positions do not average what two leave
    // out: s off by, in float32 products, two planes and three, 16 x 64 x 512, 40000 classes 9.4e-7, 2.4e-6 and below 1e-6, 4 x 256 1.4e-6, 2.2e-6 and
    // below 1e-6; but 2 x 512 1.9e-6 and (two) 2.0e-6, 4 x 1024 1.3e-6 and 1.5e-6, where two are what float32 products are.
    // us of the call, two and three: 2 x 38 x 776, 44209 classes 227 and 160; 40 x 2048, 60000 classes 305 and 368; 4 x 64 x 1024, 32000 classes 171 and
    // 195; 4 x 256: 345 and 466; 16 x 256: 1152 and 1553; 16 x 128 x 256, 30000 classes 278 and 355; where the product is small three cost nothing: 15 x
    // 127 x 192, 3958 classes 104 and 97, 4 x 512 x 1024, 4000 classes 133 and 137, but 2 x 1024 x 1000, 8000 classes 195 and 235
    L.planes = dtype == VGC_F32 ? 3u : P == 1 ? 1u : P < 512u || (uint64_t)N * V * H <= 9000000000u ? 3u : 2u;
    // samples of one position: the FC form, from planes where many rows or outputs are what it takes (us of the whole call by planes and by floats:
    // 64 x 1024, 4200 classes 57.0 and 52.8; 64 x 2048, 4000 58.9 and 66.7; 20 x 512, 9000 43.3 and 36.9; 16 x 1024, 32000 119 and 101; 32 x 4096,
    // 20000 222 and 232; 128 x 2048, 50001 442 and 684), directly where it is small (200000 outputs: 19 and by floats 21, 500000: 36 and 30), else
    // from floats
    L.sum_thin = P == 1 && N <= 256u && (uint64_t)V * H <= (256u << 10);
    L.sum_planes = P == 1 && dtype == VGC_BF16 && N >= 32u && (uint64_t)V * H >= (6u << 20) && fc_planes_supported(N, 256, H);
    const uint64_t row = 2ull * L.rows.planes * L.rows.Kp, dt = L.dx_thin ? 0 : 2ull * L.planes * L.Lq;
    const uint64_t d32 = P == 1 ? (L.sum_planes ? 16ull : 4ull) * N : 0;
    L.piece = L.dx_thin ? V : piece_of(V, row + dt + d32, 2048ull << 20);
    // large tiles where there is work for them (16000 classes, 2048 x 2048: 265 us and 277 by small ones, 512 x 4096: 160 and 158, 256 x 512:
    // 51 and 39; 4000 classes, 4096 x 4096: 257 and 287)
    L.dx_large = dtype == VGC_BF16 && L.Lq > 128u && (uint64_t)L.Lq * H * V >= 50000000000u;
    const uint64_t n = dtype == VGC_F32 ? tiles<Cut>(L.Lq, H) : L.dx_large ? tiles<Large>(L.Lq, H) : tiles<Small>(L.Lq, H);
    L.splits = 1;
    while (n * L.splits < (dtype == VGC_F32 || L.dx_large ? 256u : 512u) && L.piece / (L.splits * 2u) >= 256u && L.splits < 64u) L.splits *= 2u;
    size_t off = 0;
    L.x = off; if (!L.rows.in_place) off = align_up(off + N * row, 256);
    L.xt = off; off = align_up(off + (L.sum_planes ? fc_planes_bytes(1, N, H) : L.sum_thin ? 0 : P == 1 ? (size_t)N * H * 4 : 2 * (size_t)H * L.rows.planes * L.Lq), 256);
    L.w = off; if (!L.rows.in_place) off = align_up(off + L.piece * row, 256);
    L.d = off; if (!L.dx_thin) off = align_up(off + 2 * (size_t)L.piece * L.planes * L.Lq, 256);
    L.d32 = off; if (P == 1) off = align_up(off + 4 * (size_t)N * L.piece, 256);
    L.d2 = off; if (L.sum_planes) off += fc_planes_bytes(3, N, L.piece);
    L.out = off; if (!L.dx_thin) off += (size_t)L.splits * N * H * sizeof(float);
    off = align_up(off, 16);
    L.scales = off; if (dtype == VGC_BF16 && P > 1) off += (size_t)B * sizeof(float);
    L.rest = off; if (dtype == VGC_BF16 && !L.dx_thin) off += (size_t)N * sizeof(float);
    L.total = off;
    return L;
}
size_t softmax_loss_backward_workspace_bytes(int dtype, uint32_t B, uint32_t P, uint32_t H, uint32_t V) { return backward_plan(dtype, B, P, H, V).total; }

int launch_softmax_loss_backward(int dtype, const void* X, const void* W, const int64_t* target, const float* lse, const float* weight, uint32_t B,
                                 uint32_t P, uint32_t H, uint32_t V, float c, void* dX, float* g_out, float* s_out, void* workspace, hipStream_t stream) {
    const BackwardPlan L = backward_plan(dtype, B, P, H, V);
    const uint32_t N = B * P;
    char* ws = static_cast<char*>(workspace);
    const size_t size = dtype == VGC_F32 ? 4 : 2;
    const bool by_position = s_out && P > 1;
    int rc;
    uint16_t *xs = (uint16_t*)(ws + L.x), *xt = (uint16_t*)(ws + L.xt), *wp = (uint16_t*)(ws + L.w);
    float* out = reinterpret_cast<float*>(ws + L.out);
    LossArgs A = {};
    A.N = N; A.Lq = L.Lq;
    A.K = L.rows.in_place ? H : L.rows.Kp;
    A.at = Positions{B, P, L.Pp};
    A.target = target; A.lse = lse; A.weight = weight; A.V_all = V;
    A.scales = Scales{nullptr, P == 1};
    if (dtype == VGC_BF16 && weight) {
        A.scales.of = P == 1 ? weight : (const float*)(ws + L.scales);
        if (P > 1) {
            hipLaunchKernelGGL(k_loss_scales, dim3(B), dim3(1024), 0, stream, weight, target, P, (float*)(ws + L.scales));
            if ((rc = hip_check(hipGetLastError(), "launch k_loss_scales")) != VGC_OK) return rc;
        }
    }
    if ((dX && !L.dx_thin) || by_position) A.dt = (uint16_t*)(ws + L.d);
    A.planes = dtype == VGC_F32 || by_position ? L.planes : 1u;
    if (P == 1 && (s_out || L.dx_thin)) A.d32 = (float*)(ws + L.d32);
    if (dtype == VGC_BF16 && dX && !L.dx_thin) A.rest = (float*)(ws + L.rest);
    if (!L.rows.in_place && (rc = launch_plane_rows(dtype, {X, N, H, xs}, {}, stream)) != VGC_OK) return rc;
    A.x = matrix_of(L.rows, X, xs, N, H);
    if (by_position) {
        const dim3 grid((L.Lq + 63u) / 64u, (H + 63u) / 64u);
        if (dtype == VGC_BF16) hipLaunchKernelGGL(k_planes_columns<uint16_t>, grid, dim3(256), 0, stream, (const uint16_t*)X, target, A.at, H, L.Lq, xt);
        else hipLaunchKernelGGL(k_planes_columns<float>, grid, dim3(256), 0, stream, (const float*)X, target, A.at, H, L.Lq, xt);
        if ((rc = hip_check(hipGetLastError(), "launch k_planes_columns")) != VGC_OK) return rc;
    } else if (s_out && L.sum_planes) {
        if ((rc = launch_square_planes(dtype, X, target, N, H, xt, stream)) != VGC_OK) return rc;
    } else if (s_out && !L.sum_thin) {
        const dim3 grid((uint32_t)(((uint64_t)N * ((H + 7u) / 8u) + 255u) / 256u));
        if (dtype == VGC_F32) hipLaunchKernelGGL(k_asked_rows<float>, grid, dim3(256), 0, stream, (const float*)X, target, N, H, (float*)xt);
        else hipLaunchKernelGGL(k_asked_rows<uint16_t>, grid, dim3(256), 0, stream, (const uint16_t*)X, target, N, H, (float*)xt);
        if ((rc = hip_check(hipGetLastError(), "launch k_asked_rows")) != VGC_OK) return rc;
    }
    for (uint32_t v0 = 0; v0 < V; v0 += L.piece) {
        A.v0 = v0;
        A.V = std::min(L.piece, V - v0);
        A.plane = (uint64_t)A.V * L.Lq;
        const char* rows = static_cast<const char*>(W) + (size_t)v0 * H * size;
        if (!L.rows.in_place && (rc = launch_plane_rows(dtype, {rows, A.V, H, wp}, {}, stream)) != VGC_OK) return rc;
        A.w = matrix_of(L.rows, rows, wp, A.V, H);
        ThinArgs R = {A.w.base, A.x.base, A.w.ld, A.x.ld};
        if (dtype == VGC_F32) R = ThinArgs{rows, X, H, H};   // (as floats, also where the planes are there for dX)
        LossArgs T = A;
        if (is_thin(L.tile) && dtype == VGC_F32) T.K = H;
        if ((rc = launch_logits<false>(L.tile, dtype, R, T, stream)) != VGC_OK) return rc;
        const Matrix Dt = {A.dt, A.V, L.Lq, A.plane};
        if (dX && L.dx_thin) {
            const dim3 grid(tiles(N, kThinDx, H, kThinDx));
            if (dtype == VGC_F32) hipLaunchKernelGGL(k_loss_dx_thin<float>, grid, dim3(kThinWaves * 64), 0, stream, A.d32, (const float*)W, N, V, H, (float*)dX);
            else hipLaunchKernelGGL(k_loss_dx_thin<uint16_t>, grid, dim3(kThinWaves * 64), 0, stream, A.d32, (const uint16_t*)W, N, V, H, (uint16_t*)dX);
            if ((rc = hip_check(hipGetLastError(), "launch k_loss_dx_thin")) != VGC_OK) return rc;
        } else if (dX) {
            const uint32_t M = B * L.Pp;
            if (dtype == VGC_F32)
                hipLaunchKernelGGL(k_loss_dx<Cut>, dim3(tiles<Cut>(M, H) * L.splits), dim3(Cut::NW * 64), 0, stream, Dt, A.w, A.at, A.scales, H, L.splits, (int)(v0 > 0), out);
            else if (L.dx_large)
                hipLaunchKernelGGL(k_loss_dx<Large>, dim3(tiles<Large>(M, H) * L.splits), dim3(Large::NW * 64), 0, stream, Dt, A.w, A.at, A.scales, H, L.splits, (int)(v0 > 0), out);
            else
                hipLaunchKernelGGL(k_loss_dx<Small>, dim3(tiles<Small>(M, H) * L.splits), dim3(Small::NW * 64), 0, stream, Dt, A.w, A.at, A.scales, H, L.splits, (int)(v0 > 0), out);
            if ((rc = hip_check(hipGetLastError(), "launch k_loss_dx")) != VGC_OK) return rc;
        }
        float *g = g_out ? g_out + (size_t)v0 * H : nullptr, *s = s_out ? s_out + (size_t)v0 * H : nullptr;
        if (by_position) {
            const Matrix Xt = {xt, H, L.Lq, (uint64_t)H * L.Lq};
            // (us of the call, into the caches and past them: 33 MB of outputs 83 and 87, 114 MB 163 and 168, 262 MB 214 and 197, 983 MB 415 and 367)
            const bool past = (uint64_t)V * H * (g ? 8u : 4u) > (192ull << 20);
#define VGC_SUMS(S) do { \
                if (past) hipLaunchKernelGGL((k_loss_sums<S, true>), dim3(tiles<S>(A.V, H)), dim3(S::NW * 64), 0, stream, Dt, Xt, B, L.Pp, A.scales, c, g, s); \
                else hipLaunchKernelGGL((k_loss_sums<S, false>), dim3(tiles<S>(A.V, H)), dim3(S::NW * 64), 0, stream, Dt, Xt, B, L.Pp, A.scales, c, g, s); } while (0)
            if (dtype == VGC_F32) VGC_SUMS(CutSums);
            else if (L.planes == 3u) VGC_SUMS(SumsOfFew);
            else VGC_SUMS(Sums);
#undef VGC_SUMS
            if ((rc = hip_check(hipGetLastError(), "launch k_loss_sums")) != VGC_OK) return rc;
        } else if (s_out && L.sum_planes) {
            if ((rc = launch_square_planes(VGC_F32, A.d32, nullptr, N, A.V, ws + L.d2, stream)) != VGC_OK) return rc;
            if ((rc = launch_fc_planes(ws + L.d2, 3, xt, N, A.V, H, c, g, s, stream)) != VGC_OK) return rc;
        } else if (s_out && L.sum_thin) {
            const dim3 grid(tiles(H, 64u, A.V, 4u));
            if (dtype == VGC_F32) hipLaunchKernelGGL(k_loss_sums_thin<float>, grid, dim3(1024), 0, stream, A.d32, (const float*)X, target, N, A.V, H, c, g, s);
            else hipLaunchKernelGGL(k_loss_sums_thin<uint16_t>, grid, dim3(1024), 0, stream, A.d32, (const uint16_t*)X, target, N, A.V, H, c, g, s);
            if ((rc = hip_check(hipGetLastError(), "launch k_loss_sums_thin")) != VGC_OK) return rc;
        } else if (s_out) {
            if ((rc = launch_sqgrad(VGC_FC, VGC_F32, A.d32, xt, N, 1, A.V, H, c, g, s, nullptr, 0, stream)) != VGC_OK) return rc;
        }
    }
    if (!dX || L.dx_thin) return VGC_OK;
    const uint64_t n = (uint64_t)N * H;
    const TargetRest rest = {A.rest, target, (const uint16_t*)W, V, H};
#define VGC_JOIN(T, kWaves, per) hipLaunchKernelGGL((k_loss_dx_join<T, kWaves>), dim3((uint32_t)((n + per - 1u) / per)), dim3(kWaves == 1 ? 256 : kWaves * 64), 0, \
        stream, out, L.splits, n, rest, (T*)dX)
    if (dtype == VGC_F32) { if (L.splits >= 16u) VGC_JOIN(float, 16, 512u); else VGC_JOIN(float, 1, 2048u); }
    else { if (L.splits >= 16u) VGC_JOIN(uint16_t, 16, 512u); else VGC_JOIN(uint16_t, 1, 2048u); }
#undef VGC_JOIN
    return hip_check(hipGetLastError(), "launch k_loss_dx_join");
}

}  // namespace vgc
