// Activations kept in 8 bits for the backward pass, and the statistic formed from them.
//
// A row is cut into blocks of 32 consecutive elements; a block is stored as 32 whole numbers in -127..127 and one byte, the
// exponent of their unit, a power of two.  A value of seven bits times a power of two is a bfloat16 exactly, so what the
// statistic multiplies is the kept value itself in either type, and scaling by the unit is exact on the way in and out.
//
// Both directions are one pass, bound by memory.  Four lanes hold a block, eight elements each: one load of 16 bytes a lane
// (two for float), the maximum over four lanes without LDS, one store of 8 codes.
#include "vgc_rows.h"

namespace vgc {

constexpr int kUnits = 4;                                    // pieces of eight elements a lane has in flight
constexpr uint32_t kPiecesPerGroup = 256 * kUnits;           // pieces a workgroup takes

// Pieces are numbered row after row, `per_row` of them each (kLanes for a block: a row's last block may lack some).
// kLanes: 4, or 1 for rows of at most eight elements, which are a block by themselves.
struct PiecePlace { uint64_t row; uint32_t piece; };
struct PieceWalk {
    uint64_t row0;
    uint32_t rest, per_row;
    __device__ __forceinline__ PieceWalk(uint32_t per_row_) : per_row(per_row_) {
        const uint64_t first = (uint64_t)blockIdx.x * kPiecesPerGroup;
        row0 = first / per_row;                              // (uniform)
        rest = (uint32_t)(first - row0 * per_row);
    }
    __device__ __forceinline__ PiecePlace at(uint32_t i) const {
        const uint32_t k = rest + i, r = k / per_row;
        return PiecePlace{row0 + r, k - r * per_row};
    }
};

template <typename T, uint32_t kLanes>
__global__ __launch_bounds__(256) void k_act8_encode(const T* __restrict__ x, uint64_t R, uint32_t C, uint32_t per_row,
                                                     int8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
    const PieceWalk walk(per_row);
    PiecePlace at[kUnits];
    int n[kUnits];
    Raw8<T> raw[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        at[u] = walk.at(u * 256u + threadIdx.x);
        n[u] = at[u].row < R ? (int)C - (int)(at[u].piece * 8u) : 0;     // (0 or less: a lane past the end, whose block's others may not be)
        raw[u] = load8(x + at[u].row * C + at[u].piece * 8u, n[u], rows_at_end(at[u].row, R));
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        float f[8];
        clip8(raw[u], n[u]);
        widen8(raw[u], f);
        uint32_t top = act8_top(f);
        if (kLanes == 4) top = four_lanes_max(top);
        const uint32_t field = act8_field(top);
        if (n[u] > 0) {
            store_codes(codes + at[u].row * C + at[u].piece * 8u, act8_codes(f, field), n[u]);
            if (kLanes == 1 || (at[u].piece & 3u) == 0) exps[at[u].row * (per_row / kLanes) + at[u].piece / kLanes] = (uint8_t)field;
        }
    }
}

template <typename T, uint32_t kLanes>
__global__ __launch_bounds__(256) void k_act8_decode(const int8_t* __restrict__ codes, const uint8_t* __restrict__ exps, uint64_t R,
                                                     uint32_t C, uint32_t per_row, T* __restrict__ out) {
    const PieceWalk walk(per_row);
    PiecePlace at[kUnits];
    int n[kUnits];
    any_u2 v[kUnits];
    uint32_t field[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        at[u] = walk.at(u * 256u + threadIdx.x);
        n[u] = at[u].row < R ? (int)C - (int)(at[u].piece * 8u) : 0;
        v[u] = load_codes(codes + at[u].row * C + at[u].piece * 8u, n[u], rows_at_end(at[u].row, R));   // (what is past n is not stored)
        field[u] = n[u] > 0 ? exps[at[u].row * (per_row / kLanes) + at[u].piece / kLanes] : 0u;
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        float f[8];
        act8_values(v[u], field[u], f);
        store8(out + at[u].row * C + at[u].piece * 8u, f, n[u]);
    }
}

static uint32_t pieces_per_row(uint32_t C) { return C <= 8 ? 1u : (C + kAct8Block - 1) / kAct8Block * kAct8Lanes; }

static int act8_grid(uint64_t R, uint32_t C, const char* what, uint32_t* per_row, uint32_t* groups) {
    *per_row = pieces_per_row(C);
    const uint64_t most = 0xFFFFFFFFull / 256u;              // workgroups of a launch, which has fewer than 2^32 threads
    const uint64_t n = R > most * kPiecesPerGroup ? most + 1u : (R * *per_row + kPiecesPerGroup - 1) / kPiecesPerGroup;
    if (n > most) { set_error("%s: %llu rows of %u elements exceed the launch limit", what, (unsigned long long)R, C); return VGC_ERR_SIZE; }
    *groups = (uint32_t)n;
    return VGC_OK;
}

int launch_act8_encode(int dtype, const void* x, uint64_t R, uint32_t C, int8_t* codes, uint8_t* exps, hipStream_t stream) {
    uint32_t per_row, groups;
    const int rc = act8_grid(R, C, "vgc_act8_encode", &per_row, &groups);
    if (rc != VGC_OK) return rc;
#define VGC_LAUNCH(T, L) hipLaunchKernelGGL((k_act8_encode<T, L>), dim3(groups), dim3(256), 0, stream, (const T*)x, R, C, per_row, codes, exps)
    if (dtype == VGC_F32) { if (per_row == 1) VGC_LAUNCH(float, 1); else VGC_LAUNCH(float, 4); }
    else { if (per_row == 1) VGC_LAUNCH(uint16_t, 1); else VGC_LAUNCH(uint16_t, 4); }
#undef VGC_LAUNCH
    return hip_check(hipGetLastError(), "launch k_act8_encode");
}

int launch_act8_decode(int dtype, const int8_t* codes, const uint8_t* exps, uint64_t R, uint32_t C, void* out, hipStream_t stream) {
    uint32_t per_row, groups;
    const int rc = act8_grid(R, C, "vgc_act8_decode", &per_row, &groups);
    if (rc != VGC_OK) return rc;
#define VGC_LAUNCH(T, L) hipLaunchKernelGGL((k_act8_decode<T, L>), dim3(groups), dim3(256), 0, stream, codes, exps, R, C, per_row, (T*)out)
    if (dtype == VGC_F32) { if (per_row == 1) VGC_LAUNCH(float, 1); else VGC_LAUNCH(float, 4); }
    else { if (per_row == 1) VGC_LAUNCH(uint16_t, 1); else VGC_LAUNCH(uint16_t, 4); }
#undef VGC_LAUNCH
    return hip_check(hipGetLastError(), "launch k_act8_decode");
}

// The statistic from kept activations.  Conv form: the kept values are laid out in the type of D (exact in both) for the kernels of
// vgc_sqgrad.  FC form: bfloat16 D and the kept values as planes of values and squares (vgc_fc_planes.hip); float D and the kept values
// as floats.
struct SqgradAct8Layout { bool planes; size_t x, d, rest, rest_bytes, total; };
static SqgradAct8Layout sqgrad_act8_layout(int kind, int dtype, uint32_t B, uint32_t P, uint32_t J, uint32_t C) {
    SqgradAct8Layout L;
    const size_t rows = (size_t)B * P;
    L.planes = kind == VGC_FC && dtype == VGC_BF16;
    size_t off = 0;
    L.x = off; off += L.planes ? fc_planes_bytes(1, B, J) : align_up(rows * J * (dtype == VGC_F32 ? 4 : 2), 256);
    L.d = off; if (L.planes) off += fc_planes_bytes(1, B, C);
    L.rest = off;
    L.rest_bytes = L.planes ? 0 : sqgrad_workspace_bytes(kind, dtype, B, P, J, C);
    L.total = off + L.rest_bytes;
    return L;
}
size_t sqgrad_act8_workspace_bytes(int kind, int dtype, uint32_t B, uint32_t P, uint32_t J, uint32_t C) {
    return sqgrad_act8_layout(kind, dtype, B, P, J, C).total;
}
int launch_sqgrad_act8(int kind, int dtype, const int8_t* codes, const uint8_t* exps, const void* D, uint32_t B, uint32_t P, uint32_t J,
                       uint32_t C, float c, float* g_out, float* s_out, void* workspace, hipStream_t stream) {
    const SqgradAct8Layout L = sqgrad_act8_layout(kind, dtype, B, P, J, C);
    char* ws = static_cast<char*>(workspace);
    int rc;
    if (L.planes) {
        if ((rc = launch_square_planes_act8(codes, exps, B, J, ws + L.x, stream)) != VGC_OK) return rc;
        if ((rc = launch_square_planes(VGC_BF16, D, nullptr, B, C, ws + L.d, stream)) != VGC_OK) return rc;
        return launch_fc_planes(ws + L.x, 1, ws + L.d, B, J, C, c, g_out, s_out, stream);
    }
    if ((rc = launch_act8_decode(dtype, codes, exps, (uint64_t)B * P, J, ws + L.x, stream)) != VGC_OK) return rc;
    return launch_sqgrad(kind, dtype, ws + L.x, D, B, P, J, C, c, g_out, s_out, L.rest_bytes ? ws + L.rest : nullptr, L.rest_bytes, stream);
}

}  // namespace vgc
