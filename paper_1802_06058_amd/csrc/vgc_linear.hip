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
// Precision.  bfloat16: products are exact, sums float32; dz, which is stored in bfloat16 for the sums of W, is read so by dX's product.  float32: three planes of 8 bits an operand, rounded, six
// products of them, taken out of the instructions' sums every 32 k.
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
};
template <typename T>
__device__ __forceinline__ void finish(const Finish& F, const DropoutKey& key, uint32_t row, uint32_t col, int n, const float (&bias)[8], float (&f)[8]) {
    const size_t at = (size_t)row * F.M + col;
    Raw8<T> r;
    if (F.residual) r = load8(static_cast<const T*>(F.residual) + at, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] += bias[k];
    if (F.z) store8(static_cast<T*>(F.z) + at, f, n);
    apply_act(F.act, f);
    apply_dropout(F.drop, key, row, col / 8u, f);
    if (F.residual) {
        float g[8];
        widen8(r, g);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] += g[k];
    }
    store8(static_cast<T*>(F.y) + at, f, n);
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
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
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
                else finish<T>(A.F, key, row, col, n, bias, f);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

template <typename Shape, typename T, bool kMixed>
__global__ __launch_bounds__(Shape::NW * 64, Shape::kLds > 80 * 1024 && Shape::NW == 4 ? 1 : 2) void k_linear(LinearArgs A) {
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

// Adds the parts of k in their order, eight elements of a row a lane.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs A) {
    const uint32_t per_row = (A.F.M + 7u) / 8u;
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    if (i >= (uint64_t)A.F.N * per_row) return;
    const uint32_t row = (uint32_t)(i / per_row), col = (uint32_t)(i - (uint64_t)row * per_row) * 8u;
    const int n = (int)min(A.F.M - col, 8u);
    const float* from = A.parts + (size_t)row * A.F.M + col;
    const size_t plane = (size_t)A.F.N * A.F.M;
    float f[8] = {}, g[8], bias[8];
    bias_of(A.F, col, bias);
#pragma unroll 4
    for (uint32_t s = 0; s < A.splits; ++s) {
        widen8(load8(from + s * plane, n), g);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] += g[k];
    }
    finish<T>(A.F, dropout_key(A.F.drop), row, col, n, bias, f);
}

// ---- dz and the sums of the bias --------------------------------------------------------------------------------------------
// Workgroup (block of columns, group of rows): a team holds a row's pieces of the block, kRows of its rows in flight.  Samples of many
// positions are cut into parts, which leave a column sum each; of few, a team takes whole ones and keeps both sums.  A second kernel adds them
// in a fixed order.  Bound by memory: dy, z and dz once.
struct SlopeArgs {
    const void *dy, *z;       // z: NULL without an activation
    void* dz;
    uint16_t* planes;         // dz as operand rows of ldp where the product cannot read it as it lies, or NULL
    uint32_t ldp, count;      // planes: 1 .. 3
    float* partial;           // or NULL
    uint32_t B, P, C, lanes, blocks, parts, groups;
    bool whole;
    int act;
    Dropout drop;
};
template <typename T>
__global__ __launch_bounds__(256) void k_linear_slope(SlopeArgs A) {
    constexpr int kRows = 4;
    __shared__ float sh[2048], part[256], chan[256];
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
    Raw8<T> rd[kRows], rz[kRows];
    auto request = [&](uint32_t r0) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint32_t r = r0 + i * step;
            const int m = r < end ? n : 0;
            rd[i] = load8(static_cast<const T*>(A.dy) + (size_t)r * A.C + c0, m, rows_at_end(r, N));
            if (A.z) rz[i] = load8(static_cast<const T*>(A.z) + (size_t)r * A.C + c0, m, rows_at_end(r, N));
        }
    };
    float h[8] = {}, g[8] = {}, s[8] = {};
    uint32_t left = A.P;
    request(row);
    for (; row < end; row += kRows * step) {
        Raw8<T> nd[kRows], nz[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) { nd[i] = rd[i]; nz[i] = rz[i]; }
        if (row + kRows * step < end) request(row + kRows * step);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint32_t r = row + i * step;
            if (r >= end) continue;
            float d[8], z[8];
            clip8(nd[i], n);
            widen8(nd[i], d);
            apply_dropout(A.drop, key, r, c0 / 8u, d);
            if (A.z) {
                clip8(nz[i], n);
                widen8(nz[i], z);
                apply_slope(A.act, z, d);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] += d[k];
            if (A.whole && --left == 0u) {
                left = A.P;
#pragma unroll
                for (int k = 0; k < 8; ++k) { g[k] += h[k]; s[k] = __builtin_fmaf(h[k], h[k], s[k]); h[k] = 0.f; }
            }
            if (n > 0) store8(static_cast<T*>(A.dz) + (size_t)r * A.C + c0, d, n);
            if (A.planes && n > 0) {
                const size_t plane = (size_t)N * A.ldp;
                for (uint32_t q = 0; q < A.count; ++q) {
                    any_u4 x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = next_plane<sizeof(T) == 4>(d[2 * e], d[2 * e + 1]);
                    *reinterpret_cast<any_u4*>(A.planes + q * plane + (size_t)r * A.ldp + c0) = x;
                }
            }
        }
    }
    if (!A.partial) return;
    const uint32_t c = block * A.lanes * 8u + threadIdx.x;
    const bool mine = threadIdx.x < A.lanes * 8u && c < A.C;
    float* out = A.partial + (size_t)group * (A.whole ? 2u : 1u) * A.C + c;
    if (!A.whole) {
        channel_sums(h, A.lanes, sh, part, chan);
        if (mine) out[0] = chan[threadIdx.x];
        return;
    }
    channel_sums(g, A.lanes, sh, part, chan);
    if (mine) out[0] = chan[threadIdx.x];
    __syncthreads();
    channel_sums(s, A.lanes, sh, part, chan);
    if (mine) out[A.C] = chan[threadIdx.x];
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
//               BM   BN   WM  WN BK S PA PB
typedef TileShape<256, 256, 128, 64, 64, 2, 1, 1> Large;     // bfloat16
typedef TileShape<128, 128, 64, 64, 64, 2, 1, 1> Small;
typedef TileShape<128, 128, 64, 64, 64, 2, 1, 2> Small2;     // dX from two planes of dz
typedef TileShape<256, 128, 64, 64, 32, 2, 3, 3> Cut;        // float32

static uint32_t up8(uint32_t x) { return (x + 7u) / 8u * 8u; }
static uint64_t tiles(uint32_t a, uint32_t ta, uint32_t b, uint32_t tb) { return (uint64_t)((a + ta - 1) / ta) * ((b + tb - 1) / tb); }

enum class Tile { kLarge, kSmall, kSmall2, kCut };
// How a product [N, M] over K is formed.
struct ProductPlan { Tile tile; uint32_t splits; size_t parts; };
static ProductPlan product_plan(int dtype, uint32_t N, uint32_t M, uint32_t K, uint32_t planes_b) {
    ProductPlan L;
    L.tile = dtype == VGC_F32 ? Tile::kCut : planes_b == 2u ? Tile::kSmall2 : tiles(M, 256, N, 256) >= 192u ? Tile::kLarge : Tile::kSmall;
    const uint64_t n = L.tile == Tile::kLarge ? tiles(M, 256, N, 256) : L.tile == Tile::kCut ? tiles(M, 256, N, 128) : tiles(M, 128, N, 128);
    const uint32_t want = L.tile == Tile::kSmall ? 512u : 256u;
    L.splits = 1;
    while (n * L.splits < want && K / (L.splits * 2u) >= 256u && L.splits < 32u) L.splits *= 2u;
    L.parts = L.splits > 1u ? (size_t)L.splits * N * M * sizeof(float) : 0;
    return L;
}

template <typename T, bool kMixed>
static int launch_product(const ProductPlan& L, LinearArgs A, hipStream_t stream) {
    A.splits = L.splits;
    if (L.splits == 1u) A.parts = nullptr;
#define VGC_LAUNCH(S) hipLaunchKernelGGL((k_linear<S, T, kMixed>), dim3(tiles(A.F.M, S::BM, A.F.N, S::BN) * L.splits), dim3(S::NW * 64), 0, stream, A)
    if constexpr (sizeof(T) == 4) VGC_LAUNCH(Cut);
    else if (L.tile == Tile::kLarge) VGC_LAUNCH(Large);
    else if (L.tile == Tile::kSmall) VGC_LAUNCH(Small);
    else if constexpr (!kMixed) VGC_LAUNCH(Small2);
#undef VGC_LAUNCH
    int rc = hip_check(hipGetLastError(), "launch k_linear");
    if (rc != VGC_OK || L.splits == 1u) return rc;
    const uint64_t pieces = (uint64_t)A.F.N * ((A.F.M + 7u) / 8u);
    hipLaunchKernelGGL(k_linear_join<T>, dim3((uint32_t)((pieces + 255u) / 256u)), dim3(256), 0, stream, A);
    return hip_check(hipGetLastError(), "launch k_linear_join");
}

struct LinearPlan { ProductPlan product; bool x_there, w_there; uint32_t Kp, Cp; size_t x, w, parts, total; };
static LinearPlan linear_plan(int dtype, uint32_t N, uint32_t K, uint32_t C) {
    LinearPlan L;
    L.product = product_plan(dtype, N, C, K, 1);
    L.Kp = up8(K);
    L.Cp = up8(C);
    L.x_there = dtype == VGC_BF16 && K % 8u == 0u;
    L.w_there = dtype == VGC_BF16 && C % 8u == 0u;
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
    int rc;
    if (!L.x_there && (rc = launch_plane_rows(q.dtype, q.X, N, q.K, x, stream)) != VGC_OK) return rc;
    if (!L.w_there && (rc = launch_plane_rows(q.dtype, q.W, q.K, q.C, w, stream)) != VGC_OK) return rc;
    LinearArgs A = {};
    A.b = L.x_there ? Matrix{(const uint16_t*)q.X, N, q.K, 0} : Matrix{x, N, L.Kp, (uint64_t)N * L.Kp};
    A.a = L.w_there ? Matrix{(const uint16_t*)q.W, q.K, q.C, 0} : Matrix{w, q.K, L.Cp, (uint64_t)q.K * L.Cp};
    A.K = L.Kp;
    A.parts = (float*)(ws + L.parts);
    A.F = Finish{q.bias, q.residual, q.z, q.y, N, q.C, q.act, dropout_of(q.p, q.rng)};
    return q.dtype == VGC_F32 ? launch_product<float, true>(L.product, A, stream) : launch_product<uint16_t, true>(L.product, A, stream);
}

struct LinearBackwardPlan { ProductPlan product; bool w_there, dz_there, whole; uint32_t planes, Cp, lanes, blocks, samples_parts, groups; size_t w, dz, parts, partial, total; };
static LinearBackwardPlan linear_backward_plan(int dtype, uint32_t B, uint32_t P, uint32_t K, uint32_t C) {
    LinearBackwardPlan L;
    const uint32_t N = B * P;
    // bfloat16: a small product reads dz in two planes, 16 bits: its few sums do not average what rounding left
    const bool two = dtype == VGC_BF16 && (uint64_t)N * K * C <= (1ull << 31);
    L.planes = dtype == VGC_F32 ? 3u : two ? 2u : 1u;
    L.product = product_plan(dtype, N, K, C, L.planes);
    L.Cp = up8(C);
    L.w_there = dtype == VGC_BF16 && C % 8u == 0u;
    L.dz_there = L.w_there && !two;
    const uint32_t pieces = (C + 7u) / 8u;
    L.lanes = power_of_two(std::min(pieces, 32u));
    L.blocks = (pieces + L.lanes - 1u) / L.lanes;
    const uint32_t teams = 256u / L.lanes;
    const uint64_t want = std::max<uint64_t>(1, 2048u / L.blocks);
    L.whole = P <= 32u;
    L.samples_parts = L.whole ? 1u : (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(want / B, P / (teams * 4u)));
    L.groups = L.whole ? (uint32_t)std::min<uint64_t>(want, (B + teams - 1u) / teams) : B * L.samples_parts;
    size_t off = 0;
    L.w = off; if (!L.w_there) off = align_up(off + 2 * (size_t)(dtype == VGC_F32 ? 3 : 1) * K * L.Cp, 256);
    L.dz = off; if (!L.dz_there) off = align_up(off + 2 * (size_t)L.planes * N * L.Cp, 256);
    L.parts = off; off = align_up(off + L.product.parts, 256);
    L.partial = off; off += (size_t)L.groups * (L.whole ? 2u : 1u) * C * sizeof(float);
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
    SlopeArgs S = {q.dy, q.act == VGC_ACT_NONE ? nullptr : q.z_in, q.dz, copy ? planes : nullptr, L.Cp, L.planes, q.s_bias ? (float*)(ws + L.partial) : nullptr,
                   q.B, q.P, q.C, L.lanes, L.blocks, L.samples_parts, L.groups, L.whole, q.act, dropout_of(q.p, q.rng)};
    const dim3 grid(L.groups * L.blocks);
    if (q.dtype == VGC_F32) hipLaunchKernelGGL(k_linear_slope<float>, grid, dim3(256), 0, stream, S);
    else hipLaunchKernelGGL(k_linear_slope<uint16_t>, grid, dim3(256), 0, stream, S);
    int rc = hip_check(hipGetLastError(), "launch k_linear_slope");
    if (rc != VGC_OK) return rc;
    if (q.s_bias && (rc = launch_column_sums(S.partial, 1, L.groups, q.B, L.samples_parts, q.C, L.whole, q.c, q.g_bias, q.s_bias, nullptr, nullptr, stream)) != VGC_OK) return rc;
    if (!q.dX) return VGC_OK;
    if (!L.w_there && (rc = launch_plane_rows(q.dtype, q.W, q.K, q.C, w, stream)) != VGC_OK) return rc;
    LinearArgs A = {};
    A.a = L.w_there ? Matrix{(const uint16_t*)q.W, q.K, q.C, 0} : Matrix{w, q.K, L.Cp, (uint64_t)q.K * L.Cp};
    A.b = L.dz_there ? Matrix{(const uint16_t*)q.dz, N, q.C, 0} : Matrix{planes, N, L.Cp, (uint64_t)N * L.Cp};
    A.K = L.Cp;
    A.parts = (float*)(ws + L.parts);
    A.F = Finish{nullptr, q.residual, nullptr, q.dX, N, q.K, VGC_ACT_NONE, Dropout{nullptr, 0u, 0.f}};
    return q.dtype == VGC_F32 ? launch_product<float, false>(L.product, A, stream) : launch_product<uint16_t, false>(L.product, A, stream);
}

}  // namespace vgc
