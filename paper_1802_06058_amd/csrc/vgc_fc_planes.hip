// The FC form of the statistic from bfloat16 planes:  g = c A^T B,  s = c^2 (A.A)^T (B.B)  for rows [N, M] and [N, C] of which a row
// is a sample.  For bfloat16 values and kept 8-bit values, and for D of the softmax loss, which is float32, on one side of them.
//
// An operand enters as planes that add up to it and to its square: a bfloat16 in one plane and its square, 14 or 16 bits, in two; a float32
// in three, and its square, rounded to 24 bits, in three.  The products of the planes are exact, so g and s carry float32 sums' errors (the
// squares' third plane meets the other side's first only: 2^-25 of a product is left out); a product of squares takes four bfloat16
// instructions, or five, a quarter of the time of the float32 ones that squares in float32 need.  What is left is what the outputs take to be written, 8 bytes of each element, while N rows are
// read: 64 x (25088, 4096), g and s: 252 us by float32 instructions -> 160.  A value whose square lies below 2^-118 loses digits of it; where
// one leaves float32's range at the other end, the outputs that it reaches are formed again from the values.
#include "vgc_gemm.h"
#include "vgc_rows.h"

namespace vgc {

// What rounding to bfloat16 leaves of x (nothing where it overflows).
__device__ __forceinline__ float rest_of(float x) {
    const float hi = __uint_as_float(two_bf16(x, 0.f) << 16);
    return __builtin_isfinite(hi) ? x - hi : 0.f;
}
constexpr int square_planes(int own) { return own == 1 ? 2 : 3; }
// Planes of eight values: kOwn of the value (1: it is a bfloat16; 3), then two or three of its square.
template <int kOwn>
__device__ __forceinline__ void store_square_planes(uint16_t* out, uint64_t plane, const float (&f)[8]) {
    float rest[8], sq[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { rest[e] = f[e]; sq[e] = f[e] * f[e]; }
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        store8(out + q * plane, rest, 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) rest[e] = rest_of(rest[e]);
    }
#pragma unroll
    for (int q = 0; q < square_planes(kOwn); ++q) {
        store8(out + (kOwn + q) * plane, sq, 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) sq[e] = rest_of(sq[e]);
    }
}

// Rows of T [R, K], padded with zeros to Kp, a multiple of 8; rows with a negative target (if given) as zeros.
template <typename T, int kOwn>
__global__ __launch_bounds__(256) void k_square_planes(const T* __restrict__ src, const int64_t* __restrict__ target, uint32_t R, uint32_t K, uint32_t Kp,
                                                       uint16_t* __restrict__ dst) {
    const uint32_t per_row = Kp / 8u;
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    if (i >= (uint64_t)R * per_row) return;
    const uint64_t row = i / per_row;
    const uint32_t k = (uint32_t)(i - row * per_row) * 8u;
    float f[8] = {};
    if (!target || target[row] >= 0) widen8(load8(src + row * K + k, (int)(K - k)), f);
    store_square_planes<kOwn>(dst + row * Kp + k, (uint64_t)R * Kp, f);
}

__global__ __launch_bounds__(256) void k_square_planes_act8(const int8_t* __restrict__ codes, const uint8_t* __restrict__ exps, uint32_t R, uint32_t K,
                                                            uint32_t Kp, uint16_t* __restrict__ dst) {
    const uint32_t per_row = Kp / 8u;
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    if (i >= (uint64_t)R * per_row) return;
    const uint64_t row = i / per_row;
    const uint32_t k = (uint32_t)(i - row * per_row) * 8u;
    float f[8];
    act8_values(load_codes(codes + row * K + k, (int)(K - k)), exps[row * ((K + kAct8Block - 1) / kAct8Block) + k / kAct8Block], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = k + e < K ? f[e] : 0.f;
    store_square_planes<1>(dst + row * Kp + k, (uint64_t)R * Kp, f);
}

typedef TileShape<128, 128, 64, 64, 32, 2, 2, 2> SquareTile;
typedef TileShape<128, 128, 64, 64, 32, 2, 1, 1> RestTile;
template <int PA> using ValueTile = TileShape<128, 128, 64, 64, 32, 2, PA, 1>;

// The outputs of a wave that are not finite, from their samples' values: a square that leaves float32's range does so in planes (infinity, 0), and
// a plane's zero times infinity is NaN, whatever the sample's gradient is.  Taken as x d and (x d)^2 in float, each output is what its samples
// make it.  A lane loads a row's and a column's value of a sample; its 64 products take theirs from the other lanes.  (64 x (25088, 4096)
// with an infinity in every column: 1.9 ms; an output at a time, four loads for each of its samples, 9.9.  Where nothing but NaN is left, it ends.)
template <int PA>
__device__ __forceinline__ void form_again(const Matrix& A, const Matrix& B, uint32_t wm, uint32_t wn, uint32_t M, uint32_t C, float c, float* __restrict__ g_out,
                                           float* __restrict__ s_out) {
    typedef SquareTile Tile;
    static_assert(Tile::WM == 64 && Tile::WN == 64, "a lane for each row and column");
    const uint32_t lane = threadIdx.x & 63u, half = lane >> 5;
    const uint16_t *a = A.base + min(wm + lane, M - 1u), *b = B.base + min(wn + lane, C - 1u);
    f16v g[Tile::MT][Tile::NT] = {}, s[Tile::MT][Tile::NT] = {};
    for (uint32_t z = 0; z < A.rows; ++z) {
        float x = 0.f, d[Tile::NT];
#pragma unroll
        for (int q = PA - 1; q >= 0; --q) x += __uint_as_float((uint32_t)a[q * A.plane + (uint64_t)z * A.ld] << 16);
        const float y = __uint_as_float((uint32_t)b[(uint64_t)z * B.ld] << 16);
#pragma unroll
        for (int n = 0; n < Tile::NT; ++n) d[n] = __shfl(y, n * 32 + (lane & 31u));
        bool nothing = true;                                 // (a NaN in s is one in g)
#pragma unroll
        for (int m = 0; m < Tile::MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float r = __shfl(x, m * 32 + 8 * (i >> 2) + 4 * half + (i & 3));
#pragma unroll
                for (int n = 0; n < Tile::NT; ++n) {
                    const float p = r * d[n];
                    g[m][n][i] += p;
                    s[m][n][i] = __builtin_fmaf(p, p, s[m][n][i]);
                    nothing &= s[m][n][i] != s[m][n][i];
                }
            }
        if (__all(nothing)) break;
    }
#pragma unroll
    for (int n = 0; n < Tile::NT; ++n) {
        const uint32_t col = wn + n * 32u + (lane & 31u);
        if (col >= C) continue;
#pragma unroll
        for (int m = 0; m < Tile::MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t row = wm + m * 32u + 8u * (i >> 2) + 4u * half + (i & 3);
                if (row >= M) continue;
                float *gp = g_out ? g_out + (size_t)row * C + col : nullptr, *sp = s_out + (size_t)row * C + col;
                const float sum = s[m][n][i];
                if (gp && !__builtin_isfinite(*gp)) *gp = c * (sum == sum ? g[m][n][i] : sum);
                if (!__builtin_isfinite(*sp)) *sp = c * c * sum;
            }
    }
}

// A: PA planes of the m side, then its squares'; B: one plane of the n side, then its squares' two.
// kPast: outputs beyond what the caches hold are stored past them (64 x (25088, 4096), 822 MB: 184 us into them, 160 past them;
// 128 x (4096, 1000), 33 MB: 20 and 24).
template <int PA, bool kPast>
__global__ __launch_bounds__(SquareTile::NW * 64, 2) void k_fc_planes(Matrix A, Matrix B, uint32_t M, uint32_t C, float c, float* __restrict__ g_out,
                                                                      float* __restrict__ s_out) {
    typedef SquareTile Tile;
    static_assert(ValueTile<PA>::kLds <= Tile::kLds, "one array for all products");
    __shared__ __attribute__((aligned(1024))) uint8_t sh[Tile::kLds];
    const uint32_t tiles_n = (C + Tile::BN - 1) / Tile::BN, tiles_m = (M + Tile::BM - 1) / Tile::BM;
    const TilePlace at = in_bands(xcd_contiguous(blockIdx.x, gridDim.x), tiles_m, tiles_n);
    const uint32_t m0 = at.m * Tile::BM, n0 = at.n * Tile::BN, lane = threadIdx.x & 63u, half = lane >> 5;
    const uint32_t wm = m0 + Tile::wave_m(), wn = n0 + Tile::wave_n();
    float again = 0.f;                                       // NaN: a sum of this lane's is not finite (each looked at as it is stored: 158 -> 167 us)
    auto store = [&](const f16v (&acc)[Tile::MT][Tile::NT], float scale, float* out) {
#pragma unroll
        for (int n = 0; n < Tile::NT; ++n)
#pragma unroll
            for (int m = 0; m < Tile::MT; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) again = __builtin_fmaf(acc[m][n][i], 0.f, again);
#pragma unroll
        for (int n = 0; n < Tile::NT; ++n) {
            const uint32_t col = wn + n * 32u + (lane & 31u);
            if (col >= C) continue;
#pragma unroll
            for (int m = 0; m < Tile::MT; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t row = wm + m * 32u + 8u * (i >> 2) + 4u * half + (i & 3);
                    if (row >= M) continue;
                    float* to = out + (size_t)row * C + col;
                    if (kPast) __builtin_nontemporal_store(scale * acc[m][n][i], to);
                    else *to = scale * acc[m][n][i];
                }
        }
    };
    if (g_out) {
        f16v acc[Tile::MT][Tile::NT] = {};
        ColumnTile<ValueTile<PA>>::run(acc, sh, A, B, m0, n0, 0u, A.rows);
        store(acc, c, g_out);
    }
    f16v acc[Tile::MT][Tile::NT] = {};
    const Matrix A2 = {A.base + PA * A.plane, A.rows, A.ld, A.plane}, B2 = {B.base + B.plane, B.rows, B.ld, B.plane};
    if constexpr (square_planes(PA) == 3) {                  // (five pairs in one pass have more planes than two workgroups' LDS holds)
        const Matrix A3 = {A2.base + 2 * A.plane, A.rows, A.ld, A.plane};
        ColumnTile<RestTile>::run(acc, sh, A3, B2, m0, n0, 0u, A.rows);
    }
    ColumnTile<Tile>::run(acc, sh, A2, B2, m0, n0, 0u, A.rows);
    store(acc, c * c, s_out);
    if (__any(!(again == 0.f))) form_again<PA>(A, B, wm, wn, M, C, c, g_out, s_out);
}

// Bytes of an operand's planes: `own` of the value and those of its square.
size_t fc_planes_bytes(uint32_t own, uint32_t N, uint32_t K) { return align_up((size_t)(own + square_planes((int)own)) * N * ((K + 7u) / 8u * 8u) * 2, 256); }
// (a workgroup addresses a plane's rows with 32-bit offsets)
bool fc_planes_supported(uint32_t N, uint32_t M, uint32_t C) { return (uint64_t)(N + 64) * (M + 128ull) * 2 < 0x7FFFFFFFull && (uint64_t)(N + 64) * (C + 128ull) * 2 < 0x7FFFFFFFull; }

static dim3 planes_grid(uint32_t R, uint32_t K) { return dim3((uint32_t)(((uint64_t)R * ((K + 7u) / 8u) + 255u) / 256u)); }
int launch_square_planes_act8(const int8_t* codes, const uint8_t* exps, uint32_t R, uint32_t K, void* dst, hipStream_t stream) {
    hipLaunchKernelGGL(k_square_planes_act8, planes_grid(R, K), dim3(256), 0, stream, codes, exps, R, K, (K + 7u) / 8u * 8u, (uint16_t*)dst);
    return hip_check(hipGetLastError(), "launch k_square_planes_act8");
}
// bfloat16 rows give one plane of the value, float rows three.
int launch_square_planes(int dtype, const void* src, const int64_t* target, uint32_t R, uint32_t K, void* dst, hipStream_t stream) {
    const uint32_t Kp = (K + 7u) / 8u * 8u;
    if (dtype == VGC_BF16) hipLaunchKernelGGL((k_square_planes<uint16_t, 1>), planes_grid(R, K), dim3(256), 0, stream, (const uint16_t*)src, target, R, K, Kp, (uint16_t*)dst);
    else hipLaunchKernelGGL((k_square_planes<float, 3>), planes_grid(R, K), dim3(256), 0, stream, (const float*)src, target, R, K, Kp, (uint16_t*)dst);
    return hip_check(hipGetLastError(), "launch k_square_planes");
}
// a: planes of [N, M] with `own` planes of the value; b: planes of [N, C] with one.
int launch_fc_planes(const void* a, uint32_t own, const void* b, uint32_t N, uint32_t M, uint32_t C, float c, float* g_out, float* s_out, hipStream_t stream) {
    const uint32_t Mp = (M + 7u) / 8u * 8u, Cp = (C + 7u) / 8u * 8u;
    const Matrix A = {(const uint16_t*)a, N, Mp, (uint64_t)N * Mp}, B = {(const uint16_t*)b, N, Cp, (uint64_t)N * Cp};
    const dim3 grid(((M + 127u) / 128u) * ((C + 127u) / 128u));
    const bool past = (uint64_t)M * C * (g_out ? 8u : 4u) > (256u << 20);
#define VGC_LAUNCH(OWN, PAST) hipLaunchKernelGGL((k_fc_planes<OWN, PAST>), grid, dim3(SquareTile::NW * 64), 0, stream, A, B, M, C, c, g_out, s_out)
    if (own == 1) { if (past) VGC_LAUNCH(1, true); else VGC_LAUNCH(1, false); }
    else { if (past) VGC_LAUNCH(3, true); else VGC_LAUNCH(3, false); }
#undef VGC_LAUNCH
    return hip_check(hipGetLastError(), "launch k_fc_planes");
}

}  // namespace vgc
