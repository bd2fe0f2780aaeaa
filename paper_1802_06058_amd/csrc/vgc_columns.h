// Sums by column over the rows that a workgroup's teams take in turn.
#ifndef VGC_COLUMNS_H
#define VGC_COLUMNS_H

#include "vgc_rows.h"

namespace vgc {

// A workgroup's lanes in teams of `lanes` (a power of two): a team holds a row's pieces, a lane eight channels.  Adds v over the teams,
// by channel: chan[c] for the workgroup's 8 lanes channels.  sh: 8 floats a thread; part: a float a thread.  Ends with a barrier.
__device__ __forceinline__ void channel_sums(const float (&v)[8], uint32_t lanes, float* sh, float* part, float* chan) {
    const uint32_t tid = threadIdx.x, threads = blockDim.x, S = lanes * 8u, teams = threads / lanes;
    *reinterpret_cast<any_f4*>(sh + tid * 8u) = any_f4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<any_f4*>(sh + tid * 8u + 4u) = any_f4{v[4], v[5], v[6], v[7]};
    __syncthreads();
    if (S >= threads) {
        for (uint32_t c = tid; c < S; c += threads) {
            float sum = 0.f;
            for (uint32_t t = 0; t < teams; ++t) sum += sh[t * S + c];
            chan[c] = sum;
        }
    } else {                                                 // eight teams a thread, then the threads of a channel
        const uint32_t c = tid % S, sub = tid / S, subs = threads / S;
        float sum = 0.f;
#pragma unroll
        for (uint32_t t = 0; t < 8u; ++t) sum += sh[(sub * 8u + t) * S + c];
        part[tid] = sum;
        __syncthreads();
        if (tid < S) {
            sum = 0.f;
            for (uint32_t q = 0; q < subs; ++q) sum += part[q * S + tid];
            chan[tid] = sum;
        }
    }
    __syncthreads();
}

// Rows of `rows` that team number `team` of `teams` takes.
__device__ __forceinline__ uint32_t rows_of_team(uint32_t rows, uint32_t team, uint32_t teams) { return rows > team ? (rows - team - 1u) / teams + 1u : 0u; }

inline uint32_t power_of_two(uint32_t x) {
    uint32_t p = 1;
    while (p < x) p *= 2u;
    return p;
}

}  // namespace vgc
#endif
