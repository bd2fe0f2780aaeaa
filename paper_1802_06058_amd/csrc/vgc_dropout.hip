// Dropout over rows of C elements, y = residual + (dropped ? 0 : x / (1 - p)), with the mask drawn from a counter (vgc_epilogue.h) in
// whichever pass needs it and never stored: the backward pass is the same call on the output's gradient.
// Bound by memory: x, the residual and y once.
#include <algorithm>

#include "vgc_epilogue.h"

namespace vgc {

// A lane takes a piece of eight elements of a row; two sets of kPieces in turn, one asked for while the other is used.  kWhole: rows are whole
// pieces, and requests have no branches (past the last piece it is asked for again).  A piece's numbers are one Philox block, ten rounds, under
// which the loads lie.  16384 x 4096 bfloat16 with a residual: 81-82 us a call, 4.9 TB/s where a copy reaches 5.1; 128 x 1000 float32: 3.0 us, the launch.
template <typename T, bool kWhole, bool kResidual>
__global__ __launch_bounds__(256) void k_dropout(const T* x, const T* residual, uint32_t row0, uint32_t C, uint32_t per_row, uint32_t pieces, Dropout D, bool past, T* y) {
    constexpr int kPieces = sizeof(T) == 2 ? 4 : 2;
    const uint64_t stride = (uint64_t)gridDim.x * 256u;
    const DropoutKey key = dropout_key(D);
    struct Set { Raw8<T> a[kPieces], b[kResidual ? kPieces : 1]; };
    auto place = [&](uint64_t i, uint32_t& row, uint32_t& piece) -> size_t {
        row = (uint32_t)i / per_row;
        piece = (uint32_t)i - row * per_row;
        return (size_t)row * C + piece * 8u;
    };
    auto request = [&](Set& S, uint64_t i0) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            uint64_t i = i0 + j * stride;
            uint32_t row, piece;
            int n = 8;
            if (kWhole) i = i < pieces ? i : pieces - 1u;
            const size_t at = kWhole ? (size_t)i * 8u : place(i < pieces ? i : 0u, row, piece);
            if (!kWhole) n = i < pieces ? (int)min(C - piece * 8u, 8u) : 0;
            S.a[j] = load8(x + at, n);
            if constexpr (kResidual) S.b[j] = load8(residual + at, n);
        }
    };
    auto use = [&](const Set& S, uint64_t i0) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const uint64_t i = i0 + j * stride;
            if (i >= pieces) continue;
            uint32_t row, piece;
            const size_t at = place(i, row, piece);
            float f[8];
            widen8(S.a[j], f);
            apply_dropout(D, key, row0 + row, piece, f);
            if constexpr (kResidual) {
                float r[8];
                widen8(S.b[j], r);
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] += r[k];
            }
            store8_to(y + at, f, kWhole ? 8 : (int)min(C - piece * 8u, 8u), past);
        }
    };
    Set A, B;
    uint64_t i0 = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    request(A, i0);
    for (; i0 < pieces; i0 += 2 * kPieces * stride) {
        request(B, i0 + kPieces * stride);
        use(A, i0);
        request(A, i0 + 2 * kPieces * stride);
        use(B, i0 + kPieces * stride);
    }
}

int launch_dropout(int dtype, const void* x, const void* residual, uint32_t R, uint32_t C, const Dropout& D, void* y, hipStream_t stream) {
    const uint32_t per_row = (C + 7u) / 8u, most = std::max(1u, 0x7FFFFFFFu / per_row);     // rows a launch: pieces are counted in 32 bits
    const size_t size = dtype == VGC_F32 ? 4 : 2;
    const bool past = past_caches(y, C, (uint64_t)R * C * size * (residual ? 3u : 2u));
    for (uint32_t r = 0; r < R; r += std::min(most, R - r)) {
        const uint32_t rows = std::min(most, R - r), pieces = rows * per_row, groups = std::min((pieces + 255u) / 256u, 2048u);
        const size_t at = (size_t)r * C * size;
        const char *xs = (const char*)x + at, *rs = residual ? (const char*)residual + at : nullptr;
        char* ys = (char*)y + at;
#define VGC_LAUNCH(T, WHOLE) do { \
        if (rs) hipLaunchKernelGGL((k_dropout<T, WHOLE, true>), dim3(groups), dim3(256), 0, stream, (const T*)xs, (const T*)rs, r, C, per_row, pieces, D, past, (T*)ys); \
        else hipLaunchKernelGGL((k_dropout<T, WHOLE, false>), dim3(groups), dim3(256), 0, stream, (const T*)xs, (const T*)rs, r, C, per_row, pieces, D, past, (T*)ys); } while (0)
        if (dtype == VGC_F32) { if (C % 8u == 0u) VGC_LAUNCH(float, true); else VGC_LAUNCH(float, false); }
        else { if (C % 8u == 0u) VGC_LAUNCH(uint16_t, true); else VGC_LAUNCH(uint16_t, false); }
#undef VGC_LAUNCH
    }
    return hip_check(hipGetLastError(), "launch k_dropout");
}

}  // namespace vgc
