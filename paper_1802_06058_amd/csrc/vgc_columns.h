// Sums by column over the rows that a workgroup's teams take in turn.
#ifndef VGC_COLUMNS_H
#define VGC_COLUMNS_H

#include "vgc_rows.h"

namespace vgc {

// A workgroup's lanes in teams of `lanes` (a power of two): a team holds a row's pieces, a lane eight channels.  Adds kN vectors v over the teams,
// by channel: chan0[c], chan1[c] for the workgroup's 8 lanes channels.  sh: 8 floats a thread and vector; part: a float a thread and vector.  Ends with a barrier.
template <int kN>
__device__ __forceinline__ void channel_sums(const float (&v)[kN][8], uint32_t lanes, float* sh, float* part, float* chan0, float* chan1 = nullptr) {
    const uint32_t tid = threadIdx.x, threads = blockDim.x, S = lanes * 8u, teams = threads / lanes;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        float* to = sh + (i * threads + tid) * 8u;
        *reinterpret_cast<any_f4*>(to) = any_f4{v[i][0], v[i][1], v[i][2], v[i][3]};
        *reinterpret_cast<any_f4*>(to + 4u) = any_f4{v[i][4], v[i][5], v[i][6], v[i][7]};
    }
    __syncthreads();
    if (S >= threads) {
        for (uint32_t c = tid; c < S; c += threads)
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                float sum = 0.f;
                for (uint32_t t = 0; t < teams; ++t) sum += sh[i * threads * 8u + t * S + c];
                if (i == 0) chan0[c] = sum;
                else chan1[c] = sum;
            }
    } else {                                                 // eight teams a thread, then the threads of a channel
        const uint32_t c = tid % S, sub = tid / S, subs = threads / S;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            float sum = 0.f;
#pragma unroll
            for (uint32_t t = 0; t < 8u; ++t) sum += sh[i * threads * 8u + (sub * 8u + t) * S + c];
            part[i * threads + tid] = sum;
        }
        __syncthreads();
        for (uint32_t e = tid; e < kN * S; e += threads) {
            const uint32_t i = e / S, ch = e - i * S;
            float sum = 0.f;
            for (uint32_t q = 0; q < subs; ++q) sum += part[i * threads + q * S + ch];
            if (kN == 1 || i == 0u) chan0[ch] = sum;
            else chan1[ch] = sum;
        }
    }
    __syncthreads();
}

// A lane's pieces of the rows that its team takes: row `p` and every `step` on, below p1, of arrays of rows of C elements.  kWhole: rows are whole pieces (C % 8
// == 0), and requests have no branches, which would make a wave wait for what it asked for before: lanes past the last column take its piece again, rows past
// p1 are its last again, and neither counts.  Two sets of kRows rows are asked for in turn, one while the other is used (in one set, whose places the next
// requests take, the compiler moves registers at the loop's end, for which it waits for all of them).  Else rows come one by one, their ends element by
// element.
template <typename T, bool kWhole, int kRows, int kArrays> struct RowStream {
    const T* base[kArrays];
    uint64_t rows;            // of the arrays
    uint32_t C, p, p1, step;
    int n;
    Raw8<T> set[2][kArrays][kRows];
    __device__ __forceinline__ RowStream(const T* a, const T* b, uint32_t C, uint32_t c0, uint32_t p, uint32_t p1, uint32_t step, uint64_t rows)
        : rows(rows), C(C), p(p), p1(p1), step(step), n((int)C - (int)c0) {
        const uint32_t at = kWhole ? min(c0, C - 8u) : c0;
        base[0] = a + at;
        if (kArrays == 2) base[kArrays - 1] = b + at;
    }
    __device__ __forceinline__ Raw8<T> at(int array, uint32_t r) const {
        if (kWhole) return load8(base[array] + (uint64_t)min(r, p1 - 1u) * C, 8);
        Raw8<T> x = load8(base[array] + (uint64_t)r * C, n, rows_at_end(r, rows));
        clip8(x, n);
        return x;
    }
    __device__ __forceinline__ void request(int which, uint32_t r) {
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
            for (int a = 0; a < kArrays; ++a) set[which][a][i] = at(a, r + i * step);
    }
    __device__ __forceinline__ void begin() { if (kWhole) request(0, p); }
    template <typename Row> __device__ __forceinline__ void use(int which, uint32_t r, Row& row) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (r + i * step >= p1) continue;
            Raw8<T> x[kArrays];
#pragma unroll
            for (int a = 0; a < kArrays; ++a) x[a] = set[which][a][i];
            row(r + i * step, x);
        }
    }
    // row(r, pieces) for every row of the team, in order; after begin().
    template <typename Row> __device__ __forceinline__ void each(Row row) {
        if constexpr (kWhole) {
            for (; p < p1; p += 2 * kRows * step) {
                request(1, p + kRows * step);
                use(0, p, row);
                request(0, p + 2 * kRows * step);
                use(1, p + kRows * step, row);
            }
        } else {
            for (; p < p1; p += step) {
                Raw8<T> x[kArrays];
#pragma unroll
                for (int a = 0; a < kArrays; ++a) x[a] = at(a, p);
                row(p, x);
            }
        }
    }
};

// Rows of `rows` that team number `team` of `teams` takes.
__device__ __forceinline__ uint32_t rows_of_team(uint32_t rows, uint32_t team, uint32_t teams) { return rows > team ? (rows - team - 1u) / teams + 1u : 0u; }

inline uint32_t power_of_two(uint32_t x) {
    uint32_t p = 1;
    while (p < x) p *= 2u;
    return p;
}

}  // namespace vgc
#endif
