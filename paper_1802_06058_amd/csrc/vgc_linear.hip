// A linear layer on N rows, with what follows it, and its backward pass:
//   forward   z = X W + bias,  y = residual + drop(act(z))        X [N, K], W [K, C]
//   backward  dz = drop(dy) act'(z),  dX = add + dz W^T,  sample z's gradient of the bias  H_z = sum_p dz,  g = c sum_z H_z,  s = c^2 sum_z H_z^2
// The gradient of W needs no pass of its own here: its sums g and s are vgc_sqgrad's, from X and dz.
//
// Both products run through the loop of vgc_gemm.h with the output's columns as its m, so that a lane's results are consecutive columns of a row:
// forward, W's rows are k (MixedTile); backward, its rows are the output's columns (RowTile).  A wave turns its part in LDS, and a lane then
// finishes eight consecutive elements of a row: bias, activation, dropout and residual meet the sum while it is float32, and it is rounded once.
// Where the output has few tiles, k is shared out, and a second kernel adds the parts in a fixed order and finishes them.
//
// Precision.  bfloat16: products are exact, sums float32.  dz is stored in bfloat16, as the D that W's sums are formed from, and dX's product reads it so:
// rounded at random it leaves dX, which is rounded itself, 1.3 times as far off as its own rounding alone (2.13e-3 and 1.65e-3); two planes of it would take
// twice the matrix instructions.  Products N K C of at most 2^31, whose few sums may be further off than that, read 16 bits of it in two planes, which costs
// them nothing beside the call.  float32: three planes of 8 bits an operand, rounded, six products of them, taken out of the instructions' sums every 32 k (2e-7
// off in the root mean square); few rows are multiplied as floats.
#include <algorithm>

#include "vgc_columns.h"
#include "vgc_epilogue.h"
#include "vgc_gemm.h"
#include "vgc_planes.h"

namespace vgc {

// What becomes of a product [N, M].
struct Finish {
    const float* bias;        // or NULL, as the next two
    const void* residual;
    void* z;
    void* y;
    uint32_t N, M;
    int act;
    Dropout drop;
    bool past;                // results are stored past the caches
};
template <typename T>
__device__ __forceinline__ Raw8<T> residual_of(const Finish& F, uint32_t row, uint32_t col, int n) {
    Raw8<T> r;
    if (F.residual) r = load8(static_cast<const T*>(F.residual) + (size_t)row * F.M + col, row < F.N ? n : 0);
    return r;
}
template <typename T>
__device__ __forceinline__ void finish(const Finish& F, const DropoutKey& key, uint32_t row, uint32_t col, int n, const float (&bias)[8], const Raw8<T>& r, float (&f)[8]) {
    const size_t at = (size_t)row * F.M + col;
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] += bias[k];
    if (F.z) store8_to(static_cast<T*>(F.z) + at, f, n, F.past);
    apply_act(F.act, f);
    apply_dropout(F.drop, key, row, col / 8u, f);
    if (F.residual) {
        float g[8];
        widen8(r, g);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] += g[k];
    }
    store8_to(static_cast<T*>(F.y) + at, f, n, F.past);
}
__device__ __forceinline__ void bias_of(const Finish& F, uint32_t col, float (&bias)[8]) {
    const int n = (int)F.M - (int)col;
    if (F.bias) { widen8(load8(F.bias + col, n), bias); return; }
#pragma unroll
    for (int k = 0; k < 8; ++k) bias[k] = 0.f;
}

struct LinearArgs {
    Matrix a, b;              // a: rows are k, or the output's columns; b: rows are the output's, k contiguous
    uint32_t K, splits;
    float* parts;             // [split][N][M] where k is shared out
    Finish F;
};

// acc[mt][nt] of a wave, columns m0 + 32 mt + .. of rows n0 + 32 nt + lane % 32, through `turn`, the wave's own 32 rows of 64 columns in
// LDS.  Rows are 68 floats apart: the sixteen lanes that LDS serves together then write, and read, all of its banks once.
constexpr uint32_t kTurnPitch = 68, kTurnBytes = 32 * kTurnPitch * 4;
template <typename T, int MT, int NT>
__device__ __forceinline__ void finish_tile(f16v (&acc)[MT][NT], float* turn, uint32_t m0, uint32_t n0, uint32_t split, const LinearArgs& A) {
    static_assert(MT % 2 == 0, "columns in pairs of tiles");
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5, piece = (lane & 7u) * 8u;
    const DropoutKey key = dropout_key(A.F.drop);
#pragma unroll
    for (int mp = 0; mp < MT; mp += 2) {
        const uint32_t col = m0 + mp * 32u + piece;
        const int n = (int)A.F.M - (int)col;
        float bias[8];
        if (!A.parts) bias_of(A.F, col, bias);
        Raw8<T> res[2][4];                                   // the residual's rows, asked for 32 rows ahead
        auto ask = [&](int nt) {
            if (A.parts) return;
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q) res[nt & 1][q] = residual_of<T>(A.F, n0 + nt * 32u + q * 8u + lane / 8u, col, n);
        };
        ask(0);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt + 1 < NT) ask(nt + 1);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<f4v*>(turn + (lane & 31u) * kTurnPitch + m * 32u + 2u * i + 4u * half) =
                        f4v{acc[mp + m][nt][i], acc[mp + m][nt][i + 1], acc[mp + m][nt][i + 2], acc[mp + m][nt][i + 3]};
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q) {
                const uint32_t r = q * 8u + lane / 8u, row = n0 + nt * 32u + r;
                const f4v lo = *reinterpret_cast<const f4v*>(turn + r * kTurnPitch + piece), hi = *reinterpret_cast<const f4v*>(turn + r * kTurnPitch + piece + 4u);
                float f[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                if (row >= A.F.N || n <= 0) continue;
                if (A.parts) store8(A.parts + ((size_t)split * A.F.N + row) * A.F.M + col, f, n);
                else finish<T>(A.F, key, row, col, n, bias, res[nt & 1][q], f);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// Bound by the matrix instructions at the clock that the power limit leaves: pipes two thirds busy at 1.6-1.8 GHz of 2.4.  bfloat16, 16384 rows, us from card to
// card: 8192 to 2048 418-445, with dropout and residual 453-490 (1.12-1.21 PFLOP/s); 2048 to 8192 437-485, with gelu and z kept 523-574, since nothing of
// another tile runs beside a workgroup's end: z is 20 us of it, gelu 54; its backward product 430-480.  (Two workgroups of 256 x 128 a compute unit, whose ends
// would overlap: 477 and 551 against 460 and 536 then; four waves of 128 x 128, two thirds of the reads from LDS but one wave a SIMD: 485 and 574 against 450
// and 527.)  float32, 4096^3 by 256 x 128: 636 us, 216 TFLOP/s; by its halves, which the estimates below prefer by 1 %, 691-731.
template <typename Shape, typename T, bool kMixed>
__global__ __launch_bounds__(Shape::NW * 64, Shape::NW / 4 * (160 * 1024 / Shape::kLds)) void k_linear(LinearArgs A) {
    __shared__ __attribute__((aligned(1024))) uint8_t sh[Shape::kLds];
    static_assert(Shape::NW * kTurnBytes <= Shape::kLds, "room to turn");
    const uint32_t tiles_n = (A.F.N + Shape::BN - 1) / Shape::BN, tiles_m = (A.F.M + Shape::BM - 1) / Shape::BM;
    const uint32_t id = xcd_contiguous(blockIdx.x, gridDim.x), split = id / (tiles_m * tiles_n);
    const TilePlace at = in_bands(id - split * tiles_m * tiles_n, tiles_m, tiles_n);
    const uint32_t m0 = at.m * Shape::BM, n0 = at.n * Shape::BN, steps = (A.K + Shape::BK - 1) / Shape::BK;
    const uint32_t k0 = (uint32_t)((uint64_t)split * steps / A.splits) * Shape::BK;
    const uint32_t k1 = min((uint32_t)((uint64_t)(split + 1u) * steps / A.splits) * Shape::BK, A.K);
    f16v acc[Shape::MT][Shape::NT] = {};
    InParts<Shape, Shape::PB == 3 ? 32u : 0u> parts;
    auto after = [&](uint32_t step, int ks) { parts.after(acc, step, ks); };
    const Matrix b = {A.b.base + k0, A.b.rows, A.b.ld, A.b.plane};
    if constexpr (kMixed) {
        MixedTile<Shape>::run(acc, sh, Matrix{A.a.base + (size_t)k0 * A.a.ld, A.a.rows - k0, A.a.ld, A.a.plane}, b, m0, n0, k1 - k0, after);
    } else {
        RowTile<Shape>::run(acc, sh, Matrix{A.a.base + k0, A.a.rows, A.a.ld, A.a.plane}, b, m0, n0, Shape::BN, [](uint32_t n) { return n; }, k1 - k0, after);
    }
    parts.end(acc);
    finish_tile<T>(acc, reinterpret_cast<float*>(sh + Shape::wave() * kTurnBytes), m0 + Shape::wave_m(), n0 + Shape::wave_n(), split, A);
}

// Adds the parts of k in their order, eight elements of a row a lane.  Four parts of one row of 4096: 3.5 us, a launch's own time.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_join(Finish F, uint32_t splits, const float* __restrict__ parts) {
    const uint32_t per_row = (F.M + 7u) / 8u;
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    if (i >= (uint64_t)F.N * per_row) return;
    const uint32_t row = (uint32_t)(i / per_row), col = (uint32_t)(i - (uint64_t)row * per_row) * 8u;
    const int n = (int)min(F.M - col, 8u);
    const float* from = parts + (size_t)row * F.M + col;
    const size_t plane = (size_t)F.N * F.M;
    float f[8] = {}, g[8], bias[8];
    bias_of(F, col, bias);
#pragma unroll 4
    for (uint32_t s = 0; s < splits; ++s) {
        widen8(load8(from + s * plane, n), g);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] += g[k];
    }
    finish<T>(F, dropout_key(F.drop), row, col, n, bias, residual_of<T>(F, row, col, n), f);
}

// ---- few rows ---------------------------------------------------------------------------------------------------------------
// A workgroup of 16 waves owns 16 kV columns by 16 NT rows of the output and its waves share k, both operands straight from memory into registers.
// The instruction wants k by lane group and a row (of a) or column (of b) by lane; which k and which column a place stands for is free:
//   forward   a lane asks for kV consecutive columns of W in each of its k's rows, so that a wave's load takes whole 16 kV columns of four rows; column j
//             of the lanes is an instruction's operand (bfloat16: eight k's pairs put together by byte permutes)
//   backward  a lane asks for 16 bytes of a row of W, instruction j taking rows 16 j + lane % 16
// Rows are read where they lie (but for odd numbers of bfloat16, see product_plan).  Requests have no branches, which would make a wave wait for what it asked
// for before: past an edge a place is moved back to the last one inside, of k with the elements that others count dropped from b's, of columns and rows with
// results that others have too.
// The waves' sums meet in LDS, four lanes add an output piece's sixteen and one finishes it.
// float32 is multiplied as floats.
// Bound by what a compute unit's loads bring, whole lines of 128 bytes at some 31-41 GB/s each: 128 x 784 x 1000 float32 7.7 us; one row of bfloat16 by 4096 x
// 4096, four parts of k, 8.7 and the join (the estimates below give that size to tiles).
constexpr uint32_t kThinWaves = 16;
template <typename T> struct ThinArgs {
    const T *a, *b, *rest;    // W; the rows of X or dz, and (backward, bfloat16) what rounding left of dz
    uint32_t lda, ldb, K, splits;
    float* parts;             // [split][N][M] where k is shared out over workgroups too
    Finish F;
};
template <int kBytes> struct AnyBytes;
template <> struct AnyBytes<4> { typedef uint32_t type __attribute__((aligned(2))); };
template <> struct AnyBytes<8> { typedef any_u2 type; };
template <> struct AnyBytes<16> { typedef any_u4 type; };

// kV columns of a row.
template <typename T, int kV> struct Columns {
    static constexpr int kWords = kV * (int)sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p) {
        const typename AnyBytes<kWords * 4>::type v = *reinterpret_cast<const typename AnyBytes<kWords * 4>::type*>(p);
        if constexpr (kWords == 1) w[0] = v;
        else
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = v[i];
    }
};
template <typename T> struct ThinRow;                        // a lane's k of a row, 16 bytes; drop: the first so many do not count
template <> struct ThinRow<uint16_t> {
    static constexpr uint32_t kK = 8;
    any_u4 r;
    __device__ __forceinline__ void load(const uint16_t* p) { r = *reinterpret_cast<const any_u4*>(p); }
    __device__ __forceinline__ void drop(int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] &= n <= 2 * i ? 0xFFFFFFFFu : n == 2 * i + 1 ? 0xFFFF0000u : 0u;
    }
    __device__ __forceinline__ bf8v operand() const { return __builtin_bit_cast(bf8v, r); }
};
template <> struct ThinRow<float> {
    static constexpr uint32_t kK = 4;
    any_f4 r;
    __device__ __forceinline__ void load(const float* p) { r = *reinterpret_cast<const any_f4*>(p); }
    __device__ __forceinline__ void drop(int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = i >= n ? r[i] : 0.f;
    }
};

template <typename T, bool kMixed, int kV, int NT, bool kRest>
__global__ __launch_bounds__(kThinWaves * 64) void k_linear_thin(ThinArgs<T> A) {
    typedef ThinRow<T> Row;
    constexpr uint32_t kK = Row::kK, kStep = 4 * kK, kM = 16 * kV, kN = 16 * NT, kPitch = kM + 4;
    constexpr int kRegs = kMixed ? (int)kK * Columns<T, kV < 2 && sizeof(T) == 2 ? 2 : kV>::kWords : kV * 4;   // of a step's a
    constexpr int kAhead = kRegs + 4 * NT * (kRest ? 2 : 1) <= 16 ? 4 : 2;
    __shared__ float sh[kThinWaves][kN][kPitch];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15u, kl = (lane >> 4) * kK;
    const uint32_t tiles_n = (A.F.N + kN - 1) / kN, tiles = gridDim.x / A.splits, id = xcd_contiguous(blockIdx.x, gridDim.x);
    const uint32_t split = id / tiles, tile = id - split * tiles, m0 = tile / tiles_n * kM, n0 = tile % tiles_n * kN, M = A.F.M, K = A.K, steps = (K + kStep - 1) / kStep;
    const uint32_t begin = (uint32_t)((uint64_t)split * steps / A.splits) * kStep, end = min((uint32_t)((uint64_t)(split + 1u) * steps / A.splits) * kStep, K);
    struct Step {
        Columns<T, kV> c[kMixed ? kK : 1];
        Row w[kMixed ? 1 : kV], x[NT], rest[kRest ? NT : 1];
    };
    const T *b[NT], *rest[NT], *a[kMixed ? 1 : kV];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const size_t at = (size_t)min(n0 + t * 16u + l16, A.F.N - 1u) * A.ldb;
        b[t] = A.b + at;
        if constexpr (kRest) rest[t] = A.rest + at;
    }
    if constexpr (kMixed) {
        a[0] = A.a + min(m0 + l16 * kV, M - (uint32_t)kV);
    } else {
#pragma unroll
        for (int j = 0; j < kV; ++j) a[j] = A.a + (size_t)min(m0 + j * 16u + l16, M - 1u) * A.lda;
    }
    auto request = [&](uint32_t k0) -> Step {
        Step S;
        const uint32_t k = min(k0 + kl, K - kK);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            S.x[t].load(b[t] + k);
            if constexpr (kRest) S.rest[t].load(rest[t] + k);
        }
        if constexpr (kMixed) {
#pragma unroll
            for (uint32_t t = 0; t < kK; ++t) S.c[t].load(a[0] + (size_t)(k + t) * A.lda);
        } else {
#pragma unroll
            for (int j = 0; j < kV; ++j) S.w[j].load(a[j] + k);
        }
        return S;
    };
    f4v acc[kV][NT] = {};
    auto multiply = [&](Step& S, uint32_t k0) {
        if (k0 + kStep > K) {
            const int moved = (int)(k0 + kl) - (int)(K - kK);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                S.x[t].drop(moved);
                if constexpr (kRest) S.rest[t].drop(moved);
            }
        }
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                bf8v a;
                if constexpr (kMixed) {
                    uint32_t v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        v[u] = __builtin_amdgcn_perm(S.c[2 * u + 1].w[j / 2], S.c[2 * u].w[j / 2], j % 2 ? 0x07060302u : 0x05040100u);
                    const any_u4 q = {v[0], v[1], v[2], v[3]};
                    a = __builtin_bit_cast(bf8v, q);
                } else {
                    a = S.w[j].operand();
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if constexpr (kRest) acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, S.rest[t].operand(), acc[j][t], 0, 0, 0);
                    acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, S.x[t].operand(), acc[j][t], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < kV; ++j)
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float a;
                        if constexpr (kMixed) a = __uint_as_float(S.c[e].w[j]);
                        else a = S.w[j].r[e];
                        acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, S.x[t].r[e], acc[j][t], 0, 0, 0);
                    }
        }
    };
    constexpr uint32_t kTurn = kThinWaves * kStep;
    Step S[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (begin + wave * kStep + i * kTurn < end) S[i] = request(begin + wave * kStep + i * kTurn);
    for (uint32_t k = begin + wave * kStep; k < end; k += kAhead * kTurn)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (k + i * kTurn >= end) break;
            multiply(S[i], k + i * kTurn);
            if (k + (kAhead + i) * kTurn < end) S[i] = request(k + (kAhead + i) * kTurn);
        }
    // result r of a lane: row lane % 16 of the output's; column 4 (lane / 16) + r of instruction j
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < kV; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t q = (lane >> 4) * 4u + r, c = kMixed ? min(m0 + q * kV, M - (uint32_t)kV) + j - m0 : j * 16u + q;
                if (!kMixed || c < kM) sh[wave][t * 16 + l16][c] = acc[j][t][r];       // (a column before the workgroup's first is another's)
            }
    __syncthreads();
    constexpr uint32_t kPieces = kM / 8;
    const uint32_t piece = tid / 4u % kPieces, r = tid / 4u / kPieces, row = n0 + r, c0 = m0 + piece * 8u;
    if (r >= kN) return;
    float f[8] = {};
#pragma unroll
    for (uint32_t w = 0; w < kThinWaves / 4u; ++w) {
        const float* p = sh[(tid & 3u) * (kThinWaves / 4u) + w][r] + piece * 8u;
        const any_f4 lo = *reinterpret_cast<const any_f4*>(p), hi = *reinterpret_cast<const any_f4*>(p + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) { f[k] += lo[k]; f[4 + k] += hi[k]; }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {                            // over four lanes
        f[k] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(f[k]), 0xB1, 0xF, 0xF, false));
        f[k] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(f[k]), 0x4E, 0xF, 0xF, false));
    }
    const int n = (int)M - (int)c0;
    if ((tid & 3u) != 0u || row >= A.F.N || n <= 0) return;
    if (A.splits > 1u) { store8(A.parts + ((size_t)split * A.F.N + row) * M + c0, f, n); return; }
    float bias[8];
    bias_of(A.F, c0, bias);
    finish<T>(A.F, dropout_key(A.F.drop), row, c0, n, bias, residual_of<T>(A.F, row, c0, n), f);
}

// ---- dz and the sums of the bias --------------------------------------------------------------------------------------------
// Workgroup (block of columns, group of rows): a team holds a row's pieces of the block, kRows of its rows in flight.  Samples of many
// positions are cut into parts, which leave a column sum each; of few, a team takes whole ones and keeps both sums.  A second kernel adds them
// in a fixed order.  Bound by memory: dy, z and dz once; 16 x 1024 x 8192 bfloat16 with gelu 150-165 us, 4.9-5.4 TB/s.
struct SlopeArgs {
    const void *dy, *z;       // z: NULL without an activation
    void* dz;
    void* rest;               // like dz: what rounding left of it, or NULL
    uint16_t* planes;         // dz as operand rows of ldp where the product cannot read it as it lies, or NULL
    uint32_t ldp, count;      // planes: 1 .. 3
    float* partial;           // or NULL (no sums); one group of whole samples leaves the sums themselves:
    float *g_out, *s_out;     // (g_out or NULL)
    float c;
    uint32_t B, P, C, lanes, blocks, parts, groups;
    bool whole;
    int act;
    Dropout drop;
};
template <typename T, bool kWhole, bool kZ>
__global__ __launch_bounds__(256) void k_linear_slope(SlopeArgs A) {
    constexpr int kRows = sizeof(T) == 2 ? 4 : 2;
    __shared__ float sh[4096], part[512], chan[2][256];
    const uint32_t teams = 256u / A.lanes, team = threadIdx.x / A.lanes, block = blockIdx.x % A.blocks, group = blockIdx.x / A.blocks;
    const uint32_t c0 = (block * A.lanes + threadIdx.x % A.lanes) * 8u;
    const int n = (int)A.C - (int)c0;
    const uint32_t N = A.B * A.P;
    uint32_t row, end, step;
    if (A.whole) {
        const uint64_t t = (uint64_t)group * teams + team, all = (uint64_t)A.groups * teams;
        row = (uint32_t)(t * A.B / all) * A.P;
        end = (uint32_t)((t + 1u) * A.B / all) * A.P;
        step = 1u;
    } else {
        const uint32_t z = group / A.parts, q = group - z * A.parts;
        row = z * A.P + (uint32_t)((uint64_t)q * A.P / A.parts) + team;
        end = z * A.P + (uint32_t)((uint64_t)(q + 1u) * A.P / A.parts);
        step = teams;
    }
    const DropoutKey key = dropout_key(A.drop);
    float h[8] = {}, g[8] = {}, s[8] = {};
    uint32_t left = A.P;
    if (row < end) {
        RowStream<T, kWhole, kRows, kZ ? 2 : 1> X(static_cast<const T*>(A.dy), static_cast<const T*>(A.z), A.C, c0, row, end, step, N);
        X.begin();
        X.each([&](uint32_t r, const Raw8<T> (&in)[kZ ? 2 : 1]) {
            float d[8];
            widen8(in[0], d);
            apply_dropout(A.drop, key, r, c0 / 8u, d);
            if constexpr (kZ) {
                float z[8];
                widen8(in[1], z);
                apply_slope(A.act, z, d);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] += d[k];
            if (A.whole && --left == 0u) {
                left = A.P;
#pragma unroll
                for (int k = 0; k < 8; ++k) { g[k] += h[k]; s[k] = __builtin_fmaf(h[k], h[k], s[k]); h[k] = 0.f; }
            }
            if (n <= 0) return;
            store8(static_cast<T*>(A.dz) + (size_t)r * A.C + c0, d, n);
            if (A.rest) {
                float left_of[8];
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    const uint32_t x = two_bf16(d[k], d[k + 1]);
                    left_of[k] = d[k] - __uint_as_float(x << 16);
                    left_of[k + 1] = d[k + 1] - __uint_as_float(x & 0xFFFF0000u);
                }
                store8(static_cast<T*>(A.rest) + (size_t)r * A.C + c0, left_of, n);
            }
            if (A.planes) {
                const size_t plane = (size_t)N * A.ldp;
                for (uint32_t q = 0; q < A.count; ++q) {
                    any_u4 x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = next_plane<sizeof(T) == 4>(d[2 * e], d[2 * e + 1]);
                    *reinterpret_cast<any_u4*>(A.planes + q * plane + (size_t)r * A.ldp + c0) = x;
                }
            }
        });
    }
    if (!A.partial && !A.s_out) return;
    const uint32_t c = block * A.lanes * 8u + threadIdx.x;
    const bool mine = threadIdx.x < A.lanes * 8u && c < A.C;
    float* out = A.s_out ? nullptr : A.partial + (size_t)group * (A.whole ? 2u : 1u) * A.C + c;
    if (!A.whole) {
        const float v[1][8] = {{h[0], h[1], h[2], h[3], h[4], h[5], h[6], h[7]}};
        channel_sums<1>(v, A.lanes, sh, part, chan[0]);
        if (mine) out[0] = chan[0][threadIdx.x];
        return;
    }
    const float v[2][8] = {{g[0], g[1], g[2], g[3], g[4], g[5], g[6], g[7]}, {s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7]}};
    channel_sums<2>(v, A.lanes, sh, part, chan[0], chan[1]);
    if (!mine) return;
    if (A.s_out) {
        if (A.g_out) A.g_out[c] = A.c * chan[0][threadIdx.x];
        A.s_out[c] = A.c * A.c * chan[1][threadIdx.x];
        return;
    }
    out[0] = chan[0][threadIdx.x];
    out[A.C] = chan[1][threadIdx.x];
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
//               BM   BN   WM  WN BK S PA PB
typedef TileShape<256, 256, 64, 128, 64, 2, 1, 1> Large;     // bfloat16 (with 128 x 64 a wave 16384 x 2048 x 8192 462 us, so 448; k in steps of 32 the same)
typedef TileShape<128, 128, 64, 64, 64, 2, 1, 1> Small;      // two workgroups a compute unit
typedef TileShape<128, 128, 64, 32, 64, 4, 1, 1> Deep;       // one: what two would hide of each other's waits, four stages and two waves a SIMD have to
typedef TileShape<128, 64, 64, 32, 64, 3, 1, 1> Narrow;      // where those leave compute units idle
typedef TileShape<128, 128, 64, 32, 64, 3, 1, 2> Small2;     // dX from two planes of dz
typedef TileShape<256, 128, 64, 64, 32, 2, 3, 3> Cut;        // float32: the largest that registers and LDS hold, and, where those leave compute units idle,
typedef TileShape<128, 128, 64, 32, 32, 3, 3, 3> CutMid;     // halves
typedef TileShape<128, 64, 64, 32, 32, 4, 3, 3> CutSmall;    // and quarters of it

static uint32_t up8(uint32_t x) { return (x + 7u) / 8u * 8u; }
static uint64_t tiles(uint32_t a, uint32_t ta, uint32_t b, uint32_t tb) { return (uint64_t)((a + ta - 1) / ta) * ((b + tb - 1) / tb); }

enum class Tile { kLarge, kSmall, kSmall2, kCut, kCutMid, kCutSmall, kThin, kDeep, kNarrow };
// How a product [N, M] over K is formed: the cheapest of its forms by what they take on this card, in us (the kernels, not the call).
//   thin    workgroups in turn on 256 compute units, 3 us each and its operands' rows at 41 GB/s, where rows of x, of which a load takes 64 bytes, count twice.
//           (estimate and measured, bfloat16: 1 x 4096 x 4096 in 64 columns, four parts of k 13.8 and 11.6, whole 22 and 20; 256 x 2048 x 2048 15.8 and
//           11.5; float32: 1000^3 31 and 35, 128 x 4096 x 4096 54 and 61, 2048 x 512 x 2048 75 and 65.  Rows that share their lines take less than
//           that: one row by 4096 x 4096 goes to 128 x 64 tiles in eight parts, 11.7 by estimate, a call of 12.3-12.7)
//   tiles   in turn too, 2.5-4 us before and after a tile's steps.  bfloat16, of 64 k: 128 x 128 0.55 us a step, from two planes of dz 0.9, 128 x 64 0.4.
//           (2048^3 20 and 24, of 128 x 64 31 and 29; 512 x 4096 x 4096 in two parts 32 and 33; 512 x 2048 x 2048 20 and 17.7, of 128 x 64 15.3 and 14.6.)
//           float32, of 32 k, after the operands were laid out: 256 x 128 2.15 us a step, 128 x 128 1.05, 128 x 64 0.7.  (4096^3 647 and 636, of the
//           smaller ones 641 and 691, 841 and 830; 2048^3 119 and 136, 103 and 105, 128 and 124; 840 x 424 x 1832 44 and 40, 30 and 30, 25 and 28; in
//           thin 33 and 35)
//   large   256 x 256 tiles of bfloat16 stand beside thin alone, which takes their place where it is expected to be cheaper than 0.55 us a step.  They take 1.75,
//           but thin takes twice its estimate where its workgroups are many: a bound for which both are right would need a better estimate of thin first.
//           (with 1.75 and with 0.55: 9 x 2872 x 60896 72 and 85, 83009 x 9064 x 8 363 and 542; 48 x 131 x 128766 74 and 37, 1017955 x 2044 x 129
//           5750 and 2410)
// A long k is shared out, in thin or by tiles, where that gives idle compute units work: the second kernel that adds the parts takes 6 us and their way through
// memory.  (more workgroups than units, for a last round less empty: 8815 x 6464 x 64 float32 in four parts 130, whole 183.)
// Where both operands are laid out, one launch does it (840 x 424 x 1832 float32 27.6 -> 25.2).  Rows of an odd number of bfloat16 are laid out at whole pieces
// first: a load at an odd element takes three times as long (129 x 1331 from 4513: 90 us, from 4512 27).  Tiles are charged for layouts as the forward pass has
// them, W's by M and X's by K; backward it is K that decides for W too, and dz's planes are written by the pass before.
struct ProductPlan { Tile tile; uint32_t splits, v, t; size_t parts; };    // thin: kV and NT
static double rounds(uint64_t groups) { return (double)((groups + 255u) / 256u); }
static double join_us(uint32_t splits, uint32_t N, uint32_t M) { return splits == 1u ? 0. : 6. + (double)splits * N * M * 4e-6 / 3.; }
static double layout_us(double elements) { return 4. + elements * 2.5e-6; }
static double thin_plan(int dtype, uint32_t N, uint32_t M, uint32_t K, uint32_t planes_b, ProductPlan& best) {
    const bool f32 = dtype == VGC_F32;
    const struct { uint32_t v, t; } shapes[] = {{4, 2}, {4, 1}, {2, 2}, {2, 1}, {1, 1}};
    double least = 1e30;
    for (const auto& q : shapes) {
        if ((q.v < 2u && !f32) || (q.t == 2u && N <= 16u)) continue;
        const uint64_t n = tiles(M, 16u * q.v, N, 16u * q.t);
        if (n > (1u << 20)) continue;                        // (a launch has fewer than 2^32 threads)
        for (uint32_t splits = 1; splits <= 16u && (splits == 1u || (K / splits >= 512u && n * splits <= 2048u)); splits *= 2u) {
            const double us = rounds(n * splits) * (3. + (double)K / splits * (q.v + 2u * q.t * (f32 ? 1u : planes_b)) * (f32 ? 64. : 32.) / 41e3) + join_us(splits, N, M);
            if (us < least) { least = us; best = ProductPlan{Tile::kThin, splits, q.v, q.t, 0}; }
        }
    }
    if (!f32 && K % 2u) least += layout_us((double)N * K * (planes_b == 2u ? 0. : 1.));
    return least;
}
static ProductPlan product_plan(int dtype, uint32_t N, uint32_t M, uint32_t K, uint32_t planes_b, bool odd_w) {
    const bool f32 = dtype == VGC_F32;
    // Large tiles from 192 of them on, two small ones a compute unit, or one that is deep.  (us: 16384 x 2048 x 8192 by large tiles 448, small 566; 4096^3 113
    // and 148; 4096 x 1024 x 1024 27 and 16; 2048^3 small 31, deep 24; 4096 x 4096 x 1024 58 and 43; 8192 x 1024 x 1024 27 and 31)
    const uint64_t large = tiles(M, 256, N, 256), small = tiles(M, 128, N, 128);
    ProductPlan L, thin;
    double us = 1e30;
    auto by_tiles = [&](Tile tile, uint64_t n, uint32_t k, double start, double step) {
        for (uint32_t splits = 1; splits <= 32u && (splits == 1u || (K / splits >= 256u && n * splits <= 512u)); splits *= 2u) {
            const double t = rounds(n * splits) * (start + step * (double)((K + k - 1u) / k) / splits) + join_us(splits, N, M);
            if (t < us) { us = t; L = ProductPlan{tile, splits, 0, 0, 0}; }
        }
    };
    if (f32) {
        by_tiles(Tile::kCut, tiles(M, 256, N, 128), 32u, 2.5, 2.15);
        by_tiles(Tile::kCutMid, small, 32u, 3., 1.05);
        by_tiles(Tile::kCutSmall, tiles(M, 128, N, 64), 32u, 4., 0.7);
    } else if (planes_b == 2u) by_tiles(Tile::kSmall2, small, 64u, 2.5, 0.9);
    else if (large >= 192u) by_tiles(Tile::kLarge, large, 64u, 2.5, 0.55);
    else {
        by_tiles(small > 256u ? Tile::kSmall : Tile::kDeep, small, 64u, 2.5, 0.55);
        by_tiles(Tile::kNarrow, tiles(M, 128, N, 64), 64u, 2.5, 0.4);
    }
    us += (f32 || odd_w || M % 8u ? layout_us((double)K * M) : 0.) + (f32 || K % 8u ? layout_us((double)N * K) : 0.);
    if (K >= (f32 ? 4u : 8u) && M >= 4u) {                   // (what a place past an edge is moved back by)
        const double by_thin = thin_plan(dtype, N, M, K, planes_b, thin) + (!f32 && odd_w ? layout_us((double)K * M) : 0.);
        if (by_thin < us) L = thin;
    }
    L.parts = L.splits > 1u ? (size_t)L.splits * N * M * sizeof(float) : 0;
    return L;
}

static bool past(int dtype, uint32_t N, uint32_t M, uint32_t K, const void* z, const void* y) {
    const uint64_t bytes = ((uint64_t)N * M * (z ? 2u : 1u) + (uint64_t)N * K + (uint64_t)K * M) * (dtype == VGC_F32 ? 4u : 2u);
    return past_caches(y, M, bytes) && (!z || past_caches(z, M, bytes));
}
template <typename T>
static int launch_join(const Finish& F, uint32_t splits, float* parts, hipStream_t stream) {
    const uint64_t pieces = (uint64_t)F.N * ((F.M + 7u) / 8u);
    hipLaunchKernelGGL(k_linear_join<T>, dim3((uint32_t)((pieces + 255u) / 256u)), dim3(256), 0, stream, F, splits, parts);
    return hip_check(hipGetLastError(), "launch k_linear_join");
}

template <typename T, bool kMixed>
static int launch_product(const ProductPlan& L, LinearArgs A, hipStream_t stream) {
    A.splits = L.splits;
    if (L.splits == 1u) A.parts = nullptr;
#define VGC_LAUNCH(S) hipLaunchKernelGGL((k_linear<S, T, kMixed>), dim3(tiles(A.F.M, S::BM, A.F.N, S::BN) * L.splits), dim3(S::NW * 64), 0, stream, A)
    if constexpr (sizeof(T) == 4) {
        if (L.tile == Tile::kCut) VGC_LAUNCH(Cut);
        else if (L.tile == Tile::kCutMid) VGC_LAUNCH(CutMid);
        else VGC_LAUNCH(CutSmall);
    }
    else if (L.tile == Tile::kLarge) VGC_LAUNCH(Large);
    else if (L.tile == Tile::kSmall) VGC_LAUNCH(Small);
    else if (L.tile == Tile::kDeep) VGC_LAUNCH(Deep);
    else if (L.tile == Tile::kNarrow) VGC_LAUNCH(Narrow);
    else if constexpr (!kMixed) VGC_LAUNCH(Small2);
#undef VGC_LAUNCH
    int rc = hip_check(hipGetLastError(), "launch k_linear");
    return rc != VGC_OK || L.splits == 1u ? rc : launch_join<T>(A.F, L.splits, A.parts, stream);
}

template <typename T, bool kMixed, bool kRest>
static int launch_thin(const ProductPlan& L, ThinArgs<T> A, float* parts, hipStream_t stream) {
    A.splits = L.splits;
    A.parts = parts;
#define VGC_LAUNCH(V, NT) hipLaunchKernelGGL((k_linear_thin<T, kMixed, V, NT, kRest>), dim3(tiles(A.F.M, 16 * V, A.F.N, 16 * NT) * L.splits), dim3(kThinWaves * 64), 0, stream, A)
    if (L.t == 1u) {
        if (L.v == 4u) VGC_LAUNCH(4, 1);
        else if (L.v == 2u) VGC_LAUNCH(2, 1);
        else if constexpr (sizeof(T) == 4) VGC_LAUNCH(1, 1);
    } else {
        if (L.v == 4u) VGC_LAUNCH(4, 2);
        else VGC_LAUNCH(2, 2);
    }
#undef VGC_LAUNCH
    const int rc = hip_check(hipGetLastError(), "launch k_linear_thin");
    return rc != VGC_OK || L.splits == 1u ? rc : launch_join<T>(A.F, L.splits, parts, stream);
}

struct LinearPlan { ProductPlan product; bool x_there, w_there; uint32_t Kp, Cp; size_t x, w, parts, total; };
static LinearPlan linear_plan(int dtype, uint32_t N, uint32_t K, uint32_t C) {
    LinearPlan L;
    L.product = product_plan(dtype, N, C, K, 1, C % 2u != 0u);
    L.Kp = up8(K);
    L.Cp = up8(C);
    const bool thin = L.product.tile == Tile::kThin;
    L.x_there = (thin && dtype == VGC_F32) || (dtype == VGC_BF16 && K % (thin ? 2u : 8u) == 0u);
    L.w_there = (thin && dtype == VGC_F32) || (dtype == VGC_BF16 && C % (thin ? 2u : 8u) == 0u);
    const size_t planes = dtype == VGC_F32 ? 3 : 1;
    size_t off = 0;
    L.x = off; if (!L.x_there) off = align_up(off + 2 * planes * N * L.Kp, 256);
    L.w = off; if (!L.w_there) off = align_up(off + 2 * planes * K * L.Cp, 256);
    L.parts = off; off += L.product.parts;
    L.total = off;
    return L;
}
size_t linear_workspace_bytes(int dtype, uint32_t N, uint32_t K, uint32_t C) { return linear_plan(dtype, N, K, C).total; }

int launch_linear(const LinearCall& q, void* workspace, hipStream_t stream) {
    const uint32_t N = q.B * q.P;
    const LinearPlan L = linear_plan(q.dtype, N, q.K, q.C);
    char* ws = static_cast<char*>(workspace);
    uint16_t *x = (uint16_t*)(ws + L.x), *w = (uint16_t*)(ws + L.w);
    const Finish F = {q.bias, q.residual, q.z, q.y, N, q.C, q.act, dropout_of(q.p, q.rng), past(q.dtype, N, q.C, q.K, q.z, q.y)};
    int rc;
    const PlaneRows X = {q.X, N, q.K, x}, W = {q.W, q.K, q.C, w};
    if (!L.x_there && (rc = launch_plane_rows(q.dtype, X, L.w_there ? PlaneRows{} : W, stream)) != VGC_OK) return rc;
    if (L.x_there && !L.w_there && (rc = launch_plane_rows(q.dtype, W, {}, stream)) != VGC_OK) return rc;
    float* parts = (float*)(ws + L.parts);
    if (L.product.tile == Tile::kThin) {
        if (q.dtype == VGC_F32)
            return launch_thin<float, true, false>(L.product, ThinArgs<float>{(const float*)q.W, (const float*)q.X, nullptr, q.C, q.K, q.K, 1, nullptr, F}, parts, stream);
        const ThinArgs<uint16_t> T = {L.w_there ? (const uint16_t*)q.W : w, L.x_there ? (const uint16_t*)q.X : x, nullptr, L.w_there ? q.C : L.Cp, L.x_there ? q.K : L.Kp, q.K, 1, nullptr, F};
        return launch_thin<uint16_t, true, false>(L.product, T, parts, stream);
    }
    LinearArgs A = {};
    A.b = L.x_there ? Matrix{(const uint16_t*)q.X, N, q.K, 0} : Matrix{x, N, L.Kp, (uint64_t)N * L.Kp};
    A.a = L.w_there ? Matrix{(const uint16_t*)q.W, q.K, q.C, 0} : Matrix{w, q.K, L.Cp, (uint64_t)q.K * L.Cp};
    A.K = L.Kp;
    A.parts = parts;
    A.F = F;
    return q.dtype == VGC_F32 ? launch_product<float, true>(L.product, A, stream) : launch_product<uint16_t, true>(L.product, A, stream);
}

struct LinearBackwardPlan { ProductPlan product; bool w_there, dz_there, rest, whole, direct; uint32_t planes, Cp, lanes, blocks, samples_parts, groups; size_t w, dz, parts, partial, total; };
static LinearBackwardPlan linear_backward_plan(int dtype, uint32_t B, uint32_t P, uint32_t K, uint32_t C) {
    LinearBackwardPlan L;
    const uint32_t N = B * P;
    // bfloat16: a small product reads dz in two planes, 16 bits: its few sums do not average what rounding left
    const bool two = dtype == VGC_BF16 && (uint64_t)N * K * C <= (1ull << 31);
    L.planes = dtype == VGC_F32 ? 3u : two ? 2u : 1u;
    L.product = product_plan(dtype, N, K, C, dtype == VGC_F32 ? 1u : L.planes, C % 2u != 0u);
    L.Cp = up8(C);
    const bool thin = L.product.tile == Tile::kThin;
    L.w_there = (thin && dtype == VGC_F32) || (dtype == VGC_BF16 && C % (thin ? 2u : 8u) == 0u);
    L.dz_there = L.w_there && (thin || !two);
    L.rest = L.dz_there && two;
    const uint32_t pieces = (C + 7u) / 8u;
    L.lanes = power_of_two(std::min(pieces, 32u));
    L.blocks = (pieces + L.lanes - 1u) / L.lanes;
    const uint32_t teams = 256u / L.lanes;
    // Samples whole or in parts, whichever leaves a team fewer rows in turn, counted over rounds of 1024 workgroups: a round takes some 3 us and 0.3 a row (16
    // samples of 32 x 512: whole, one team each, 16.7 us, in parts 5.2).  The second kernel takes 4.5, without which one group of workgroups of 32 teams can do
    // where it has few samples (128 x 1000 to 1000 float32, the whole call 17.1 -> 13.9).
    auto us = [&](uint64_t groups, uint64_t rows) { return (double)((groups * L.blocks + 1023u) / 1024u) * (3. + 0.3 * (double)rows); };
    const uint64_t want = std::max<uint64_t>(1, 2048u / L.blocks), whole_groups = std::min<uint64_t>(want, (B + teams - 1u) / teams);
    const uint64_t parts = std::max<uint64_t>(1, std::min<uint64_t>(want / B, P / (teams * 2u)));
    const double whole_us = us(whole_groups, P * ((B + whole_groups * teams - 1u) / (whole_groups * teams))), parts_us = us(B * parts, (P + parts * teams - 1u) / (parts * teams));
    L.whole = whole_us <= parts_us;
    L.samples_parts = L.whole ? 1u : (uint32_t)parts;
    L.groups = L.whole ? (uint32_t)whole_groups : B * L.samples_parts;
    const uint32_t narrow = std::min(L.lanes, 8u), narrow_blocks = (pieces + narrow - 1u) / narrow;
    L.direct = (double)((narrow_blocks + 1023u) / 1024u) * (3. + 0.3 * (double)P * (double)((B + 256u / narrow - 1u) / (256u / narrow))) <= std::min(whole_us, parts_us) + 4.5;
    if (L.direct) { L.lanes = narrow; L.blocks = narrow_blocks; L.whole = true; L.samples_parts = L.groups = 1u; }
    size_t off = 0;
    L.w = off; if (!L.w_there) off = align_up(off + 2 * (size_t)(dtype == VGC_F32 ? 3 : 1) * K * L.Cp, 256);
    L.dz = off; if (!L.dz_there) off = align_up(off + 2 * (size_t)L.planes * N * L.Cp, 256);
    if (L.rest) off = align_up(off + 2 * (size_t)N * C, 256);    // (in dz's place)
    L.parts = off; off = align_up(off + L.product.parts, 256);
    L.partial = off; if (!L.direct) off += (size_t)L.groups * (L.whole ? 2u : 1u) * C * sizeof(float);
    L.total = off;
    return L;
}
size_t linear_backward_workspace_bytes(int dtype, uint32_t B, uint32_t P, uint32_t K, uint32_t C) { return linear_backward_plan(dtype, B, P, K, C).total; }

int launch_linear_backward(const LinearCall& q, void* workspace, hipStream_t stream) {
    const uint32_t N = q.B * q.P;
    const LinearBackwardPlan L = linear_backward_plan(q.dtype, q.B, q.P, q.K, q.C);
    char* ws = static_cast<char*>(workspace);
    uint16_t *w = (uint16_t*)(ws + L.w), *planes = (uint16_t*)(ws + L.dz);
    const bool copy = q.dX && !L.dz_there;
    SlopeArgs S = {q.dy, q.act == VGC_ACT_NONE ? nullptr : q.z_in, q.dz, q.dX && L.rest ? planes : nullptr, copy ? planes : nullptr, L.Cp, L.planes, q.s_bias && !L.direct ? (float*)(ws + L.partial) : nullptr,
                   L.direct ? q.g_bias : nullptr, L.direct ? q.s_bias : nullptr, q.c, q.B, q.P, q.C, L.lanes, L.blocks, L.samples_parts, L.groups, L.whole, q.act, dropout_of(q.p, q.rng)};
    const dim3 grid(L.groups * L.blocks);
#define VGC_LAUNCH(T, WHOLE) do { if (S.z) hipLaunchKernelGGL((k_linear_slope<T, WHOLE, true>), grid, dim3(256), 0, stream, S); \
        else hipLaunchKernelGGL((k_linear_slope<T, WHOLE, false>), grid, dim3(256), 0, stream, S); } while (0)
    if (q.dtype == VGC_F32) { if (q.C % 8u == 0u) VGC_LAUNCH(float, true); else VGC_LAUNCH(float, false); }
    else { if (q.C % 8u == 0u) VGC_LAUNCH(uint16_t, true); else VGC_LAUNCH(uint16_t, false); }
#undef VGC_LAUNCH
    int rc = hip_check(hipGetLastError(), "launch k_linear_slope");
    if (rc != VGC_OK) return rc;
    if (q.s_bias && !L.direct && (rc = launch_column_sums(S.partial, 1, L.groups, q.B, L.samples_parts, q.C, L.whole, q.c, q.g_bias, q.s_bias, nullptr, nullptr, stream)) != VGC_OK) return rc;
    if (!q.dX) return VGC_OK;
    const Finish F = {nullptr, q.residual, nullptr, q.dX, N, q.K, VGC_ACT_NONE, Dropout{nullptr, 0u, 0.f}, past(q.dtype, N, q.K, q.C, nullptr, q.dX)};
    if (!L.w_there && (rc = launch_plane_rows(q.dtype, {q.W, q.K, q.C, w}, {}, stream)) != VGC_OK) return rc;
    float* parts = (float*)(ws + L.parts);
    if (L.product.tile == Tile::kThin) {
        if (q.dtype == VGC_F32)
            return launch_thin<float, false, false>(L.product, ThinArgs<float>{(const float*)q.W, (const float*)q.dz, nullptr, q.C, q.C, q.C, 1, nullptr, F}, parts, stream);
        const uint32_t ld = L.w_there ? q.C : L.Cp;
        const ThinArgs<uint16_t> T = {L.w_there ? (const uint16_t*)q.W : w, L.dz_there ? (const uint16_t*)q.dz : planes, L.dz_there ? planes : planes + (size_t)N * L.Cp, ld, ld, q.C, 1, nullptr, F};
        return L.planes == 2u ? launch_thin<uint16_t, false, true>(L.product, T, parts, stream) : launch_thin<uint16_t, false, false>(L.product, T, parts, stream);
    }
    LinearArgs A = {};
    A.a = L.w_there ? Matrix{(const uint16_t*)q.W, q.K, q.C, 0} : Matrix{w, q.K, L.Cp, (uint64_t)q.K * L.Cp};
    A.b = L.dz_there ? Matrix{(const uint16_t*)q.dz, N, q.C, 0} : Matrix{planes, N, L.Cp, (uint64_t)N * L.Cp};
    A.K = L.Cp;
    A.parts = parts;
    A.F = F;
    return q.dtype == VGC_F32 ? launch_product<float, false>(L.product, A, stream) : launch_product<uint16_t, false>(L.product, A, stream);
}

void linear_form(int dtype, bool backward, uint32_t B, uint32_t P, uint32_t K, uint32_t C, uint32_t* form) {
    ProductPlan L;
    form[4] = 1u;
    if (backward) {
        const LinearBackwardPlan q = linear_backward_plan(dtype, B, P, K, C);
        L = q.product;
        form[4] = q.planes;
    } else {
        L = linear_plan(dtype, B * P, K, C).product;
    }
    form[0] = (uint32_t)L.tile; form[1] = L.splits; form[2] = L.v; form[3] = L.t;
}

}  // namespace vgc
