// Softmax cross entropy of a linear layer over many classes, without its logits:
//   z[n, v] = sum_h X[n, h] W[v, h],   lse[n] = log sum_v exp z[n, v],   loss[n] = lse[n] - z[n, t_n]
//   backward  D[n, v] = w_n (exp(z[n, v] - lse[n]) - [v = t_n]),   dX = D W,
//             sample z's gradient of W  G_z = sum_p D[z, p, :]^T X[z, p, :],   g = c sum_z G_z,   s = c^2 sum_z G_z . G_z
//
// Forward, the logits of a tile stay in the accumulators: a token's column of them is reduced to its maximum and the sum of the
// exponentials relative to it, and these pairs are joined over the tiles of the vocabulary by a second, small kernel.  W is the A
// operand, so that a lane's 16 results of an instruction are 16 classes of one token: the reduction is in registers but for one
// exchange between the lane halves.
// Backward, the logits are formed again, a piece of the vocabulary at a time, and D of the piece goes to the workspace in the
// two orders in which the two products that follow read it with k contiguous; memory is bounded by the piece, not by the
// vocabulary.  All three products run through the one loop of vgc_gemm.h.
//
// Precision.  bfloat16 inputs: products are exact, sums float32.  D is rounded to bfloat16 for dX, which is rounded to bfloat16
// itself; for g and s, which are float32, it is kept in two pieces, 16 significant bits.  float32 inputs: every operand is cut
// exactly into three pieces of 8 bits and a product is formed from the six pairs of pieces that reach 2^-24 of it: the pieces lie
// one after another along k (smallest products first), so that the same loop runs over six times the length.
#include <algorithm>

#include "vgc_gemm.h"
#include "vgc_rows.h"

namespace vgc {

// ---- operands -------------------------------------------------------------------------------------------------------------
// A float cut into three bfloat16 pieces, largest first, by truncation: 8 + 8 + 8 bits, exact (but for bits below the smallest
// subnormal).  The pieces of an operand follow each other along k in slots, and slot i of the one side meets slot i of the other:
// the six pairs of pieces whose product reaches 2^-24 of the whole, the smallest first.
constexpr uint32_t kSlotsF32 = 6;
__device__ constexpr int kPieceA[6] = {2, 0, 1, 1, 0, 0}, kPieceB[6] = {0, 2, 1, 0, 1, 0};
struct Cut3 { uint32_t p[3]; };                              // each the upper half of a float's bits
__device__ __forceinline__ Cut3 cut3(float x) {
    Cut3 c;
    c.p[0] = __float_as_uint(x) >> 16;
    const bool finite = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
    if (!finite && (__float_as_uint(x) & 0x7FFFFFu)) c.p[0] |= 0x40u;        // (a NaN keeps being one without its low bits)
    const float r1 = finite ? x - __uint_as_float(c.p[0] << 16) : 0.f;
    c.p[1] = __float_as_uint(r1) >> 16;
    const float r2 = r1 - __uint_as_float(c.p[1] << 16);
    c.p[2] = __float_as_uint(r2) >> 16;
    return c;
}
// A gradient in two pieces rounded to nearest: within 2^-18 of it.
__device__ __forceinline__ float bf16_round(float x) { return __uint_as_float(two_bf16(x, 0.f) << 16); }

__device__ __forceinline__ uint32_t bits16(float x) { return __float_as_uint(x) >> 16; }     // of a value that is a bfloat16

// Rows as they are, padded to whole pieces of 8 (dst rows are slots * Kp long).
template <typename T, bool kSecond>
__global__ __launch_bounds__(256) void k_slots_rows(const T* __restrict__ src, uint32_t R, uint32_t K, uint32_t Kp, uint16_t* __restrict__ dst) {
    const uint32_t per_row = Kp / 8u;
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    if (i >= (uint64_t)R * per_row) return;
    const uint64_t row = i / per_row;
    const uint32_t k = (uint32_t)(i - row * per_row) * 8u;
    float f[8];
    widen8(load8(src + row * K + k, (int)(K - k)), f);
    constexpr uint32_t slots = sizeof(T) == 4 ? kSlotsF32 : 1u;
    uint16_t* out = dst + row * slots * Kp + k;
    if (sizeof(T) == 2) {
        store8(out, f, 8);
        return;
    }
    Cut3 c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = cut3(f[e]);
#pragma unroll
    for (uint32_t s = 0; s < slots; ++s) {
        const int q = kSecond ? kPieceB[s] : kPieceA[s];
        any_u4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = c[2 * e].p[q] | c[2 * e + 1].p[q] << 16;
        *reinterpret_cast<any_u4*>(out + (size_t)s * Kp) = v;
    }
}

// Columns as rows, for the second side: dst[k][(z slots + s) Pp + p] = piece of src[z P + p][k], zero for p in [P, Pp) and for
// rows that are not asked for (target given and negative).  slots: 6 for float; 1, or 2 times the same for the two pieces of D.
// A workgroup turns 64 positions by 64 columns in LDS.
template <typename T>
__global__ __launch_bounds__(256) void k_slots_columns(const T* __restrict__ src, const int64_t* __restrict__ target, uint32_t B, uint32_t P,
                                                       uint32_t Pp, uint32_t K, uint32_t slots, uint32_t ld, uint16_t* __restrict__ dst) {
    __shared__ float t[64][65];
    const uint32_t k0 = blockIdx.y * 64u, q0 = blockIdx.x * 64u, total = B * Pp;
    const uint32_t col = threadIdx.x & 63u, r4 = threadIdx.x >> 6;
#pragma unroll 4
    for (uint32_t r = r4; r < 64u; r += 4u) {
        const uint32_t q = q0 + r, z = q / Pp, p = q - z * Pp;
        float x = 0.f;
        if (q < total && p < P && k0 + col < K) {
            const uint64_t row = (uint64_t)z * P + p;
            if (!target || target[row] >= 0) {
                if (sizeof(T) == 4) x = ((const float*)src)[row * K + k0 + col];
                else x = __uint_as_float((uint32_t)((const uint16_t*)src)[row * K + k0 + col] << 16);
            }
        }
        t[r][col] = x;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t u = threadIdx.x; u < 512u; u += 256u) {
        const uint32_t kk = u >> 3, q = q0 + (u & 7u) * 8u;
        if (k0 + kk >= K || q >= total) continue;
        const uint32_t z = q / Pp, p = q - z * Pp;           // (Pp is a multiple of 8: the eight belong to one sample)
        uint16_t* out = dst + (size_t)(k0 + kk) * ld + (size_t)z * slots * Pp + p;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = t[(u & 7u) * 8u + e][kk];
        if (sizeof(T) == 2) {
            for (uint32_t s = 0; s < slots; ++s) store8(out + (size_t)s * Pp, f, 8);
        } else {
            Cut3 c[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = cut3(f[e]);
#pragma unroll
            for (uint32_t s = 0; s < kSlotsF32; ++s) {
                any_u4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = c[2 * e].p[kPieceB[s]] | c[2 * e + 1].p[kPieceB[s]] << 16;
                *reinterpret_cast<any_u4*>(out + (size_t)s * Pp) = v;
            }
        }
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

__global__ __launch_bounds__(256) void k_clear(uint4* p, uint64_t n) {
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    if (i < n) p[i] = make_uint4(0u, 0u, 0u, 0u);
}

// ---- the logits of a tile and what becomes of them --------------------------------------------------------------------------
struct LossArgs {
    Rows w, x;                // classes [v0, v0 + V) and tokens
    uint32_t K, V, N;
    int64_t v0;
    const int64_t* target;
    // forward
    float2* partial;          // [block][N]: maximum, sum of exponentials relative to it
    float* picked;            // the target's logit
    uint32_t block0;
    // backward
    int64_t V_all;
    const float *lse, *weight;
    uint16_t *d, *dt;         // D by tokens, rows of slots * Vp; by classes, rows of ld_dt, sample z's slot s at (z slots + s) Pp
    float* d32;               // D in float by tokens, rows of V
    uint32_t Vp, ld_dt, P, Pp;
};

constexpr float kLog2e = 1.44269504088896341f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// acc[mt][nt] of a wave: classes m0 + 32 mt + .., tokens n0 + 32 nt + lane % 32.
template <int MT, int NT>
__device__ __forceinline__ void finish_forward(f16v (&acc)[MT][NT], uint32_t m0, uint32_t n0, const LossArgs& A) {
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5;
    const float kNone = -__builtin_inff();
    if (m0 + MT * 32u > A.V) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (m0 + m * 32u + 8u * (i >> 2) + 4u * half + (i & 3) >= A.V)
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
                if (at == m * 32u + 8u * (i >> 2) + 4u * half + (i & 3)) z_t = z;
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

template <bool kF32, int MT, int NT>
__device__ __forceinline__ void finish_backward(f16v (&acc)[MT][NT], uint32_t m0, uint32_t n0, const LossArgs& A) {
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5;
    constexpr uint32_t slots = kF32 ? kSlotsF32 : 1u, slots_t = kF32 ? kSlotsF32 : 2u;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t token = n0 + n * 32u + (lane & 31u);
        if (token >= A.N) continue;
        const int64_t t = A.target[token];
        const float lse = A.lse[token];
        float w = A.weight ? A.weight[token] : 1.f;
        if (t >= A.V_all) w = __uint_as_float(0x7FC00000u);  // not a class: the gradients say so
        const bool asked = t >= 0;
        const int64_t tl = t - A.v0;
        const uint32_t at = asked && tl >= 0 && tl < (int64_t)A.V ? (uint32_t)tl : 0xFFFFFFFFu;
        const uint32_t z = token / A.P, p = token - z * A.P;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t v = m0 + m * 32u + 8u * g + 4u * half;        // four consecutive classes
                float d[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float q = exp_of(acc[m][n][4 * g + e] - lse) - (v + e == at ? 1.f : 0.f);
                    d[e] = asked && v + e < A.V ? q * w : 0.f;
                }
                if (A.d32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (v + e < A.V) A.d32[(size_t)token * A.V + v + e] = d[e];
                }
                Cut3 c[4];
                float hi[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (kF32) c[e] = cut3(d[e]);
                    else hi[e] = bf16_round(d[e]);
                }
                if (A.d && v < A.Vp) {
                    uint16_t* out = A.d + (size_t)token * slots * A.Vp + v;
#pragma unroll
                    for (uint32_t s = 0; s < slots; ++s) {
                        uint2 o;
                        if (kF32) o = make_uint2(c[0].p[kPieceA[s]] | c[1].p[kPieceA[s]] << 16, c[2].p[kPieceA[s]] | c[3].p[kPieceA[s]] << 16);
                        else o = make_uint2(two_bf16(d[0], d[1]), two_bf16(d[2], d[3]));
                        *reinterpret_cast<uint2*>(out + (size_t)s * A.Vp) = o;
                    }
                }
                if (A.dt) {
                    const size_t col = (size_t)z * slots_t * A.Pp + p;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (v + e >= A.V) continue;
                        uint16_t* out = A.dt + (size_t)(v + e) * A.ld_dt + col;
#pragma unroll
                        for (uint32_t s = 0; s < slots_t; ++s)
                            out[(size_t)s * A.Pp] = (uint16_t)(kF32 ? c[e].p[kPieceA[s]] : bits16(s ? hi[e] : bf16_round(d[e] - hi[e])));
                    }
                }
            }
    }
}

template <typename Tile, bool kForward, bool kF32>
__global__ __launch_bounds__(Tile::NW * 64, Tile::NW == 8 ? 2 : 2) void k_logits(LossArgs A) {
    __shared__ __attribute__((aligned(1024))) uint8_t sh[Tile::kLds];
    const uint32_t tiles_n = (A.N + Tile::BN - 1) / Tile::BN, id = xcd_contiguous(blockIdx.x, gridDim.x);
    const uint32_t m0 = id / tiles_n * Tile::BM, n0 = id % tiles_n * Tile::BN;
    f16v acc[Tile::MT][Tile::NT] = {};
    Tile::template run<false>(acc, sh, A.w, A.x, m0, n0, 0u, A.K, [](uint32_t) {});
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = m0 + wave / (Tile::BN / Tile::WN) * Tile::WM, wn = n0 + wave % (Tile::BN / Tile::WN) * Tile::WN;
    if (kForward) { if (wm < A.V) finish_forward(acc, wm, wn, A); }
    else finish_backward<kF32>(acc, wm, wn, A);
}

// Few tokens, or few classes: a workgroup of eight waves owns 32 classes by 64 tokens and its waves share k in steps of 64, with
// both operands straight from memory into registers; the waves' sums meet in LDS.  In a step a lane takes the 32 consecutive k of
// its half: which k an instruction's place stands for is free as long as both operands agree.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const Rows& R, uint32_t row0, uint32_t count) {
    const uint32_t left = row0 < R.rows ? min(R.rows - row0, count) : 0u;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(R.base + (size_t)row0 * R.ld), 0, (int)(left * R.ld * 2u), 0x00020000);
}
constexpr uint32_t kThinM = 32, kThinN = 64, kThinWaves = 8;
template <bool kForward, bool kF32>
__global__ __launch_bounds__(kThinWaves * 64) void k_logits_thin(LossArgs A) {
    __shared__ float sh[kThinWaves][32][64];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tiles_n = (A.N + kThinN - 1) / kThinN, id = xcd_contiguous(blockIdx.x, gridDim.x);
    const uint32_t m0 = id / tiles_n * kThinM, n0 = id % tiles_n * kThinN;
    const __amdgpu_buffer_rsrc_t rw = rows_buffer(A.w, m0, kThinM), rx = rows_buffer(A.x, n0, kThinN);
    const uint32_t kl = (lane >> 5) * 32u, offW = ((lane & 31u) * A.w.ld + kl) * 2u, offX = ((lane & 31u) * A.x.ld + kl) * 2u;
    const uint32_t second = 32u * A.x.ld * 2u;
    struct Step { i4v w[4], x[2][4]; };
    auto request = [&](uint32_t k) -> Step {
        Step S;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t outside = k + kl + j * 8u < A.K ? 0u : 0xFFFFFFFFu, add = (k + j * 8u) * 2u;
            S.w[j] = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)((offW + add) | outside), 0, 0));
            S.x[0][j] = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(rx, (int)((offX + add) | outside), 0, 0));
            S.x[1][j] = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(rx, (int)((offX + second + add) | outside), 0, 0));
        }
        return S;
    };
    f16v sum[2] = {};
    Step S = request(wave * kStepK);
    for (uint32_t k = wave * kStepK; k < A.K; k += kThinWaves * kStepK) {
        const Step next = request(k + kThinWaves * kStepK);  // (past the end: zeros, not used)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < 2; ++n)
                sum[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8v, S.w[j]), __builtin_bit_cast(bf8v, S.x[n][j]), sum[n], 0, 0, 0);
        S = next;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) sh[wave][n * 16 + i][lane] = sum[n][i];
    __syncthreads();
    if (wave >= 2u) return;
    f16v acc[1][1] = {};
    for (uint32_t q = 0; q < kThinWaves; ++q)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[0][0][i] += sh[q][wave * 16u + i][lane];
    if (kForward) finish_forward(acc, m0, n0 + wave * 32u, A);
    else finish_backward<kF32>(acc, m0, n0 + wave * 32u, A);
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
// Part `split` of the sum over the piece's k, added to what the pieces before have left in the part's own plane.
template <typename Tile>
__global__ __launch_bounds__(Tile::NW * 64, 2) void k_loss_dx(Rows D, Rows Wt, uint32_t K, uint32_t splits, int add, float* __restrict__ planes) {
    __shared__ __attribute__((aligned(1024))) uint8_t sh[Tile::kLds];
    const uint32_t N = D.rows, H = Wt.rows, tiles_n = (H + Tile::BN - 1) / Tile::BN, tiles_m = (N + Tile::BM - 1) / Tile::BM;
    const uint32_t id = xcd_contiguous(blockIdx.x, gridDim.x), split = id / (tiles_n * tiles_m), tile = id - split * tiles_n * tiles_m;
    const uint32_t m0 = tile / tiles_n * Tile::BM, n0 = tile % tiles_n * Tile::BN;
    const uint32_t steps = (K + kStepK - 1) / kStepK;
    const uint32_t k0 = (uint32_t)((uint64_t)split * steps / splits) * kStepK, k1 = min((uint32_t)((uint64_t)(split + 1u) * steps / splits) * kStepK, K);
    f16v acc[Tile::MT][Tile::NT] = {};
    Tile::template run<false>(acc, sh, D, Wt, m0, n0, k0, k1, [](uint32_t) {});
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = m0 + wave / (Tile::BN / Tile::WN) * Tile::WM, wn = n0 + wave % (Tile::BN / Tile::WN) * Tile::WN;
    float* out = planes + (size_t)split * N * H;
#pragma unroll
    for (int n = 0; n < Tile::NT; ++n) {
        const uint32_t h = wn + n * 32u + (lane & 31u);
        if (h >= H) continue;
#pragma unroll
        for (int m = 0; m < Tile::MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t token = wm + m * 32u + 8u * (i >> 2) + 4u * half + (i & 3);
                if (token >= N) continue;
                float* at = out + (size_t)token * H + h;
                *at = acc[m][n][i] + (add ? *at : 0.f);
            }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_loss_dx_join(const float* __restrict__ planes, uint32_t splits, uint64_t n, T* __restrict__ dX) {
    const uint64_t i = ((uint64_t)blockIdx.x * 256u + threadIdx.x) * 8u;
    if (i >= n) return;
    const int m = n - i >= 8u ? 8 : (int)(n - i);
    float f[8], g[8];
    widen8(load8(planes + i, m), f);
    for (uint32_t s = 1; s < splits; ++s) {
        widen8(load8(planes + s * n + i, m), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] += g[e];
    }
    store8(dX + i, f, m);
}

// ---- g and s ------------------------------------------------------------------------------------------------------------------
// k runs over the samples, `seg` of it each; at a sample's end its product is squared into s, added into g, and cleared.
typedef GemmTile<128, 128, 64, 64> TileSums;
template <bool kFine>
__global__ __launch_bounds__(TileSums::NW * 64, 2) void k_loss_sums(Rows Dt, Rows Xt, uint32_t K, uint32_t seg, float c, float* __restrict__ g_out,
                                                                    float* __restrict__ s_out) {
    typedef TileSums Tile;
    __shared__ __attribute__((aligned(1024))) uint8_t sh[Tile::kLds];
    const uint32_t V = Dt.rows, H = Xt.rows, tiles_n = (H + Tile::BN - 1) / Tile::BN;
    const uint32_t id = xcd_contiguous(blockIdx.x, gridDim.x), m0 = id / tiles_n * Tile::BM, n0 = id % tiles_n * Tile::BN;
    f16v acc[Tile::MT][Tile::NT] = {}, g[Tile::MT][Tile::NT] = {}, s[Tile::MT][Tile::NT] = {};
    uint32_t left = seg;
    Tile::template run<kFine>(acc, sh, Dt, Xt, m0, n0, 0u, K, [&](uint32_t) {
        left -= kFine ? 16u : kStepK;
        if (left != 0u) return;
        left = seg;
#pragma unroll
        for (int m = 0; m < Tile::MT; ++m)
#pragma unroll
            for (int n = 0; n < Tile::NT; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = acc[m][n][i];
                    g[m][n][i] += x;
                    s[m][n][i] = __builtin_fmaf(x, x, s[m][n][i]);
                    acc[m][n][i] = 0.f;
                }
    });
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = m0 + wave / (Tile::BN / Tile::WN) * Tile::WM, wn = n0 + wave % (Tile::BN / Tile::WN) * Tile::WN;
#pragma unroll
    for (int n = 0; n < Tile::NT; ++n) {
        const uint32_t h = wn + n * 32u + (lane & 31u);
        if (h >= H) continue;
#pragma unroll
        for (int m = 0; m < Tile::MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t v = wm + m * 32u + 8u * (i >> 2) + 4u * half + (i & 3);
                if (v >= V) continue;
                if (g_out) g_out[(size_t)v * H + h] = c * g[m][n][i];
                s_out[(size_t)v * H + h] = c * c * s[m][n][i];
            }
    }
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
typedef GemmTile<256, 256, 128, 64> TileLarge;
typedef GemmTile<128, 128, 64, 64> TileSmall;
enum class LogitsTile { kLarge, kSmall, kThin };

static uint32_t up8(uint32_t x) { return (x + 7u) / 8u * 8u; }
static uint32_t tiles(uint32_t a, uint32_t ta, uint32_t b, uint32_t tb) { return (a + ta - 1) / ta * ((b + tb - 1) / tb); }

static LogitsTile logits_tile(uint32_t V, uint32_t N) {
    if (N > 128u && tiles(V, 256, N, 256) >= 192u) return LogitsTile::kLarge;
    if (N > 64u && tiles(V, 128, N, 128) >= 192u) return LogitsTile::kSmall;
    return LogitsTile::kThin;
}
static uint32_t logits_block(LogitsTile t) { return t == LogitsTile::kLarge ? 128u : t == LogitsTile::kSmall ? 64u : 32u; }

template <bool kForward, bool kF32>
static int launch_logits(LogitsTile t, const LossArgs& A, hipStream_t stream) {
    if (t == LogitsTile::kLarge)
        hipLaunchKernelGGL((k_logits<TileLarge, kForward, kF32>), dim3(tiles(A.V, 256, A.N, 256)), dim3(512), 0, stream, A);
    else if (t == LogitsTile::kSmall)
        hipLaunchKernelGGL((k_logits<TileSmall, kForward, kF32>), dim3(tiles(A.V, 128, A.N, 128)), dim3(256), 0, stream, A);
    else
        hipLaunchKernelGGL((k_logits_thin<kForward, kF32>), dim3(tiles(A.V, kThinM, A.N, kThinN)), dim3(512), 0, stream, A);
    return hip_check(hipGetLastError(), "launch k_logits");
}

// An operand's rows are used where they lie if they are bfloat16 and whole pieces of 16 bytes.
static bool rows_in_place(int dtype, uint32_t H) { return dtype == VGC_BF16 && H % 8u == 0; }
static uint32_t row_slots(int dtype) { return dtype == VGC_F32 ? kSlotsF32 : 1u; }

static int launch_rows(int dtype, bool second, const void* src, uint32_t R, uint32_t K, uint16_t* dst, hipStream_t stream) {
    const uint32_t Kp = up8(K);
    const dim3 grid((uint32_t)(((uint64_t)R * (Kp / 8u) + 255u) / 256u));
    if (dtype == VGC_BF16) hipLaunchKernelGGL((k_slots_rows<uint16_t, false>), grid, dim3(256), 0, stream, (const uint16_t*)src, R, K, Kp, dst);
    else if (second) hipLaunchKernelGGL((k_slots_rows<float, true>), grid, dim3(256), 0, stream, (const float*)src, R, K, Kp, dst);
    else hipLaunchKernelGGL((k_slots_rows<float, false>), grid, dim3(256), 0, stream, (const float*)src, R, K, Kp, dst);
    return hip_check(hipGetLastError(), "launch k_slots_rows");
}
static int launch_columns(int dtype, const void* src, const int64_t* target, uint32_t B, uint32_t P, uint32_t Pp, uint32_t K, uint32_t slots,
                          uint16_t* dst, hipStream_t stream) {
    const dim3 grid((uint32_t)(((uint64_t)B * Pp + 63u) / 64u), (K + 63u) / 64u);
    if (dtype == VGC_BF16)
        hipLaunchKernelGGL(k_slots_columns<uint16_t>, grid, dim3(256), 0, stream, (const uint16_t*)src, target, B, P, Pp, K, slots, B * slots * Pp, dst);
    else
        hipLaunchKernelGGL(k_slots_columns<float>, grid, dim3(256), 0, stream, (const float*)src, target, B, P, Pp, K, slots, B * slots * Pp, dst);
    return hip_check(hipGetLastError(), "launch k_slots_columns");
}

// The vocabulary in pieces of equal size, multiples of 256 classes, `bytes` of working memory a class.
static uint32_t piece_of(uint32_t V, uint64_t bytes, uint64_t budget) {
    uint64_t most = budget / std::max<uint64_t>(bytes, 1) / 256u * 256u;
    most = std::min<uint64_t>(std::max<uint64_t>(most, 256u), 1u << 20);
    const uint32_t pieces = (uint32_t)((V + most - 1) / most);
    return ((V + pieces - 1) / pieces + 255u) / 256u * 256u;
}

struct ForwardPlan { LogitsTile tile; uint32_t Kp, slots, piece, blocks; bool in_place; size_t x, w, partial, picked, total; };
static ForwardPlan forward_plan(int dtype, uint32_t N, uint32_t H, uint32_t V) {
    ForwardPlan L;
    L.in_place = rows_in_place(dtype, H);
    L.slots = row_slots(dtype);
    L.Kp = up8(H);
    const uint64_t row = 2ull * L.slots * L.Kp;
    L.piece = L.in_place ? V : std::min(piece_of(V, row, 256ull << 20), V);
    L.tile = logits_tile(L.piece, N);
    L.blocks = (V + logits_block(L.tile) - 1) / logits_block(L.tile);
    size_t off = 0;
    L.x = off; if (!L.in_place) off = align_up(off + N * row, 256);
    L.w = off; if (!L.in_place) off = align_up(off + L.piece * row, 256);
    L.partial = off; off = align_up(off + (size_t)L.blocks * N * sizeof(float2), 256);
    L.picked = off; off += (size_t)N * sizeof(float);
    L.total = off;
    return L;
}
size_t softmax_loss_workspace_bytes(int dtype, uint32_t N, uint32_t H, uint32_t V) { return forward_plan(dtype, N, H, V).total; }

int launch_softmax_loss(int dtype, const void* X, const void* W, const int64_t* target, uint32_t N, uint32_t H, uint32_t V, float* loss, float* lse,
                        void* workspace, hipStream_t stream) {
    const ForwardPlan L = forward_plan(dtype, N, H, V);
    char* ws = static_cast<char*>(workspace);
    const size_t size = dtype == VGC_F32 ? 4 : 2;
    int rc;
    LossArgs A = {};
    A.N = N; A.K = L.slots * L.Kp;
    A.target = target;
    A.partial = reinterpret_cast<float2*>(ws + L.partial);
    A.picked = reinterpret_cast<float*>(ws + L.picked);
    uint16_t *xs = reinterpret_cast<uint16_t*>(ws + L.x), *wsl = reinterpret_cast<uint16_t*>(ws + L.w);
    if (!L.in_place && (rc = launch_rows(dtype, true, X, N, H, xs, stream)) != VGC_OK) return rc;
    A.x = Rows{L.in_place ? (const uint16_t*)X : xs, N, A.K};
    for (uint32_t v0 = 0; v0 < V; v0 += L.piece) {
        A.v0 = v0;
        A.V = std::min(L.piece, V - v0);
        const char* rows = static_cast<const char*>(W) + (size_t)v0 * H * size;
        if (!L.in_place && (rc = launch_rows(dtype, false, rows, A.V, H, wsl, stream)) != VGC_OK) return rc;
        A.w = Rows{L.in_place ? (const uint16_t*)rows : wsl, A.V, A.K};
        A.block0 = v0 / logits_block(L.tile);
        if ((rc = launch_logits<true, false>(L.tile, A, stream)) != VGC_OK) return rc;
    }
    hipLaunchKernelGGL(k_loss_join, dim3((N + 63) / 64), dim3(1024), 0, stream, A.partial, A.picked, target, L.blocks, N, (int64_t)V, loss, lse);
    return hip_check(hipGetLastError(), "launch k_loss_join");
}

struct BackwardPlan {
    LogitsTile tile;
    uint32_t Kp, slots, slots_t, piece, Vp, Pp, splits;
    bool in_place, dx_large;
    size_t x, xt, w, wt, d, dt, planes, total;
};
static BackwardPlan backward_plan(int dtype, uint32_t B, uint32_t P, uint32_t H, uint32_t V) {
    BackwardPlan L;
    const uint32_t N = B * P;
    L.in_place = rows_in_place(dtype, H);
    L.slots = row_slots(dtype);
    L.slots_t = dtype == VGC_F32 ? kSlotsF32 : 2u;
    L.Kp = up8(H);
    // a sample's end falls on a whole step of 64 k (bfloat16: two slots of 32 positions), or, for short samples, of 16
    L.Pp = P == 1 ? 1u : P <= 24u ? up8(P) : (P + 31u) / 32u * 32u;
    const uint64_t row = 2ull * L.slots * L.Kp;
    const uint64_t per_class = (L.in_place ? 0 : row) + row + 2ull * L.slots * N + (P == 1 ? 4ull * N : 2ull * L.slots_t * B * L.Pp);
    L.piece = std::min(piece_of(V, per_class, 512ull << 20), V);
    L.Vp = up8(L.piece);
    L.tile = logits_tile(L.piece, N);
    L.dx_large = tiles(N, 256, H, 256) >= 256u;
    const uint32_t k = L.slots * L.Vp, n = L.dx_large ? tiles(N, 256, H, 256) : tiles(N, 128, H, 128);
    L.splits = 1;
    while (n * L.splits < (L.dx_large ? 256u : 512u) && k / (L.splits * 2u) >= 256u && L.splits < 64u) L.splits *= 2u;
    size_t off = 0;
    L.x = off; if (!L.in_place) off = align_up(off + N * row, 256);
    L.xt = off; off = align_up(off + (P == 1 ? (size_t)N * H * 4 : 2 * (size_t)H * L.slots_t * B * L.Pp), 256);
    L.w = off; if (!L.in_place) off = align_up(off + L.piece * row, 256);
    L.wt = off; off = align_up(off + 2 * (size_t)H * L.slots * L.Vp, 256);
    L.d = off; off = align_up(off + 2 * (size_t)N * L.slots * L.Vp, 256);
    L.dt = off; off = align_up(off + (P == 1 ? 4 * (size_t)N * L.piece : 2 * (size_t)L.piece * L.slots_t * B * L.Pp), 256);
    L.planes = off; off += (size_t)L.splits * N * H * sizeof(float);
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
    uint16_t *xs = (uint16_t*)(ws + L.x), *xt = (uint16_t*)(ws + L.xt), *wsl = (uint16_t*)(ws + L.w), *wt = (uint16_t*)(ws + L.wt);
    float* planes = reinterpret_cast<float*>(ws + L.planes);
    LossArgs A = {};
    A.N = N; A.K = L.slots * L.Kp;
    A.target = target; A.lse = lse; A.weight = weight; A.V_all = V;
    A.P = P; A.Pp = L.Pp; A.ld_dt = L.slots_t * B * L.Pp;
    if (dX) A.d = (uint16_t*)(ws + L.d);
    if (by_position) A.dt = (uint16_t*)(ws + L.dt);
    else if (s_out) A.d32 = (float*)(ws + L.dt);
    if (!L.in_place && (rc = launch_rows(dtype, true, X, N, H, xs, stream)) != VGC_OK) return rc;
    A.x = Rows{L.in_place ? (const uint16_t*)X : xs, N, A.K};
    if (by_position) {
        if ((rc = launch_columns(dtype, X, target, B, P, L.Pp, H, L.slots_t, xt, stream)) != VGC_OK) return rc;
        if (L.Pp != P) {                                     // positions that do not exist: what they meet in X is zero too, but has to be finite
            const uint64_t n = 2ull * L.piece * A.ld_dt / 16u;
            hipLaunchKernelGGL(k_clear, dim3((uint32_t)((n + 255u) / 256u)), dim3(256), 0, stream, reinterpret_cast<uint4*>(A.dt), n);
            if ((rc = hip_check(hipGetLastError(), "launch k_clear")) != VGC_OK) return rc;
        }
    } else if (s_out) {
        const dim3 grid((uint32_t)(((uint64_t)N * ((H + 7u) / 8u) + 255u) / 256u));
        if (dtype == VGC_F32) hipLaunchKernelGGL(k_asked_rows<float>, grid, dim3(256), 0, stream, (const float*)X, target, N, H, (float*)xt);
        else hipLaunchKernelGGL(k_asked_rows<uint16_t>, grid, dim3(256), 0, stream, (const uint16_t*)X, target, N, H, (float*)xt);
        if ((rc = hip_check(hipGetLastError(), "launch k_asked_rows")) != VGC_OK) return rc;
    }
    for (uint32_t v0 = 0; v0 < V; v0 += L.piece) {
        A.v0 = v0;
        A.V = std::min(L.piece, V - v0);
        A.Vp = up8(A.V);
        const char* rows = static_cast<const char*>(W) + (size_t)v0 * H * size;
        if (!L.in_place && (rc = launch_rows(dtype, false, rows, A.V, H, wsl, stream)) != VGC_OK) return rc;
        A.w = Rows{L.in_place ? (const uint16_t*)rows : wsl, A.V, A.K};
        rc = dtype == VGC_F32 ? launch_logits<false, true>(L.tile, A, stream) : launch_logits<false, false>(L.tile, A, stream);
        if (rc != VGC_OK) return rc;
        if (dX) {
            if ((rc = launch_columns(dtype, rows, nullptr, 1, A.V, A.Vp, H, L.slots, wt, stream)) != VGC_OK) return rc;
            const Rows D = {A.d, N, L.slots * A.Vp}, Wt = {wt, H, L.slots * A.Vp};
            if (L.dx_large)
                hipLaunchKernelGGL(k_loss_dx<TileLarge>, dim3(tiles(N, 256, H, 256) * L.splits), dim3(512), 0, stream, D, Wt, D.ld, L.splits, (int)(v0 > 0), planes);
            else
                hipLaunchKernelGGL(k_loss_dx<TileSmall>, dim3(tiles(N, 128, H, 128) * L.splits), dim3(256), 0, stream, D, Wt, D.ld, L.splits, (int)(v0 > 0), planes);
            if ((rc = hip_check(hipGetLastError(), "launch k_loss_dx")) != VGC_OK) return rc;
        }
        float *g = g_out ? g_out + (size_t)v0 * H : nullptr, *s = s_out ? s_out + (size_t)v0 * H : nullptr;
        if (by_position) {
            const Rows Dt = {A.dt, A.V, A.ld_dt}, Xt = {xt, H, A.ld_dt};
            const uint32_t seg = L.slots_t * L.Pp;
            const dim3 grid(tiles(A.V, TileSums::BM, H, TileSums::BN));
            if (seg % kStepK == 0) hipLaunchKernelGGL(k_loss_sums<false>, grid, dim3(256), 0, stream, Dt, Xt, A.ld_dt, seg, c, g, s);
            else hipLaunchKernelGGL(k_loss_sums<true>, grid, dim3(256), 0, stream, Dt, Xt, A.ld_dt, seg, c, g, s);
            if ((rc = hip_check(hipGetLastError(), "launch k_loss_sums")) != VGC_OK) return rc;
        } else if (s_out) {
            if ((rc = launch_sqgrad(VGC_FC, VGC_F32, A.d32, xt, N, 1, A.V, H, c, g, s, nullptr, 0, stream)) != VGC_OK) return rc;
        }
    }
    if (!dX) return VGC_OK;
    const uint64_t n = (uint64_t)N * H;
    const dim3 grid((uint32_t)((n + 2047u) / 2048u));
    if (dtype == VGC_F32) hipLaunchKernelGGL(k_loss_dx_join<float>, grid, dim3(256), 0, stream, planes, L.splits, n, (float*)dX);
    else hipLaunchKernelGGL(k_loss_dx_join<uint16_t>, grid, dim3(256), 0, stream, planes, L.splits, n, (uint16_t*)dX);
    return hip_check(hipGetLastError(), "launch k_loss_dx_join");
}

}  // namespace vgc
