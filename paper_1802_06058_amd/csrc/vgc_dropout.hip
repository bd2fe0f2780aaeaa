// Dropout over rows of C elements, y = residual + (dropped ? 0 : x / (1 - p)), with the mask drawn from a counter (vgc_epilogue.h) in
// whichever pass needs it and never stored: the backward pass is the same call on the output's gradient.
// Bound by memory: x, the residual and y once.
#include <algorithm>

#include "vgc_epilogue.h"

namespace vgc {

// A lane takes a piece of eight elements of a row, kPieces of them in flight.
template <typename T>
__global__ __launch_bounds__(256) void k_dropout(const T* x, const T* residual, uint32_t row0, uint32_t R, uint32_t C, uint32_t per_row, uint32_t pieces,
                                                 Dropout D, T* y) {
    constexpr int kPieces = 4;
    const uint32_t stride = gridDim.x * 256u;
    const DropoutKey key = dropout_key(D);
    for (uint64_t i0 = (uint64_t)blockIdx.x * 256u + threadIdx.x; i0 < pieces; i0 += (uint64_t)kPieces * stride) {
        Raw8<T> a[kPieces], b[kPieces];
        uint32_t row[kPieces], piece[kPieces];
        int n[kPieces];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const uint64_t i = i0 + (uint64_t)j * stride;
            n[j] = 0;
            row[j] = piece[j] = 0u;
            if (i >= pieces) continue;
            row[j] = (uint32_t)i / per_row;
            piece[j] = (uint32_t)i - row[j] * per_row;
            n[j] = (int)min(C - piece[j] * 8u, 8u);
            const size_t at = (size_t)row[j] * C + piece[j] * 8u;
            a[j] = load8(x + at, n[j]);
            if (residual) b[j] = load8(residual + at, n[j]);
        }
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            if (n[j] == 0) continue;
            float f[8], r[8];
            widen8(a[j], f);
            apply_dropout(D, key, row0 + row[j], piece[j], f);
            if (residual) {
                widen8(b[j], r);
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] += r[k];
            }
            store8(y + (size_t)row[j] * C + piece[j] * 8u, f, n[j]);
        }
    }
}

int launch_dropout(int dtype, const void* x, const void* residual, uint32_t R, uint32_t C, const Dropout& D, void* y, hipStream_t stream) {
    const uint32_t per_row = (C + 7u) / 8u, most = std::max(1u, 0x7FFFFFFFu / per_row);     // rows a launch: pieces are counted in 32 bits
    const size_t size = dtype == VGC_F32 ? 4 : 2;
    for (uint32_t r = 0; r < R; r += std::min(most, R - r)) {
        const uint32_t rows = std::min(most, R - r), pieces = rows * per_row, groups = std::min((pieces + 255u) / 256u, 4096u);
        const size_t at = (size_t)r * C * size;
        const char *xs = (const char*)x + at, *rs = residual ? (const char*)residual + at : nullptr;
        char* ys = (char*)y + at;
        if (dtype == VGC_F32) hipLaunchKernelGGL(k_dropout<float>, dim3(groups), dim3(256), 0, stream, (const float*)xs, (const float*)rs, r, rows, C, per_row, pieces, D, (float*)ys);
        else hipLaunchKernelGGL(k_dropout<uint16_t>, dim3(groups), dim3(256), 0, stream, (const uint16_t*)xs, (const uint16_t*)rs, r, rows, C, per_row, pieces, D, (uint16_t*)ys);
    }
    return hip_check(hipGetLastError(), "launch k_dropout");
}

}  // namespace vgc
