// Matrix products of rows with rows: C[m, n] = sum_k A[m, k] B[n, k], bfloat16 operands with k contiguous, float32 accumulators.
//
// A workgroup owns a BM x BN tile of C, a wave a WM x WN part of it in 32 x 32 tiles of v_mfma_f32_32x32x16_bf16.  Steps of 64 k
// travel from global memory straight into LDS (buffer loads with the LDS modifier: lane l of a wave-wide load deposits its 16
// bytes at M0 + 16 l), one step ahead of the one being multiplied.  A staged row is 128 bytes, eight pieces of 16; piece q of row
// r lies at place q ^ (r % 8), so that the eight rows that eight lanes read a piece of start in different banks.  The exchange is
// made on the way in by choosing which global piece each lane fetches, and on the way out in the fragment addresses.
//
// Lane l of the instruction holds, for row m = l % 32, the eight k = 8 (l / 32) .. + 7: one piece.  Its 16 results are
// C[m = 8 (i / 4) + 4 (l / 32) + i % 4][n = l % 32], i = 0..15.
#ifndef VGC_GEMM_H
#define VGC_GEMM_H

#include "vgc_internal.h"

namespace vgc {

typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef int i4v __attribute__((ext_vector_type(4)));

constexpr uint32_t kStepK = 64;

// Rows of an operand: element (row, k) at base[row * ld + k].  base and ld: multiples of 16 bytes.  A tile's rows have to span
// less than 2^32 bytes.
struct Rows {
    const uint16_t* base;
    uint32_t rows, ld;
};

// 16 bytes a lane from the bounded buffer `rsrc` (byte offset voff) to LDS byte address lds + 16 * lane.  Lanes outside the range
// deposit zeros.  Counted by vmcnt.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"              // m0 is named as clobbered on purpose
__device__ __forceinline__ void piece_to_lds(uint32_t lds, uint32_t voff, i4v rsrc) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(lds), "v"(voff), "s"(rsrc) : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ i4v rows_rsrc(const Rows& R, uint32_t row0, uint32_t count) {
    const uint64_t addr = reinterpret_cast<uint64_t>(R.base) + (uint64_t)row0 * R.ld * 2u;
    const uint32_t left = row0 < R.rows ? min(R.rows - row0, count) : 0u;
    i4v r;                                                   // uniform values; the asm operand must be scalar registers
    r[0] = (int)__builtin_amdgcn_readfirstlane((uint32_t)addr);
    r[1] = (int)__builtin_amdgcn_readfirstlane((uint32_t)(addr >> 32) & 0xFFFFu);
    r[2] = (int)__builtin_amdgcn_readfirstlane(left * R.ld * 2u);
    r[3] = 0x00020000;
    return r;
}

// Logical number of a workgroup so that each of the eight XCDs, which take workgroups in turn, gets a contiguous range: those
// that share operand rows share an L2.
__device__ __forceinline__ uint32_t xcd_contiguous(uint32_t id, uint32_t total) {
    const uint32_t per = total / 8u, rem = total % 8u, xcd = id % 8u, slot = id / 8u;
    return xcd * per + min(xcd, rem) + slot;
}

template <int kBM, int kBN, int kWM, int kWN> struct GemmTile {
    static constexpr int BM = kBM, BN = kBN, WM = kWM, WN = kWN;
    static constexpr int NW = (BM / WM) * (BN / WN), MT = WM / 32, NT = WN / 32;
    static constexpr uint32_t kABytes = BM * 128, kBBytes = BN * 128, kStage = kABytes + kBBytes;
    static constexpr uint32_t kLds = 2 * kStage + 1024;      // (the last KiB: see run)
    static_assert((BM / 8) % NW == 0 && (BN / 8) % NW == 0, "every wave issues the same loads");

    // acc += A[m0 .. , k] B[n0 .. , k] over k in [k0, k1) (multiples of 8, k0 of 64).  sh: kLds bytes.  after(k): called with
    // the k up to which acc is complete, after every 16 (kFine) or 64 of them.
    template <bool kFine, typename After>
    static __device__ __forceinline__ void run(f16v (&acc)[MT][NT], uint8_t* sh, const Rows& A, const Rows& B, uint32_t m0, uint32_t n0,
                                               uint32_t k0, uint32_t k1, After after) {
        const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t wm = wave / (BN / WN), wn = wave % (BN / WN);
        const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)sh);
        const i4v ra = rows_rsrc(A, m0, BM), rb = rows_rsrc(B, n0, BN);
        // load j of a wave covers rows 8 (j NW + wave) .. + 7 of an operand
        const uint32_t piece = (lane & 7u) ^ (lane >> 3), kl = piece * 8u;
        constexpr int kLoadsA = BM / 8 / NW, kLoadsB = BN / 8 / NW;
        const uint32_t voffA = ((wave * 8u + (lane >> 3)) * A.ld + kl) * 2u, voffB = ((wave * 8u + (lane >> 3)) * B.ld + kl) * 2u;
        const uint32_t stepA = NW * 8u * A.ld * 2u, stepB = NW * 8u * B.ld * 2u;
        auto issue = [&](uint32_t stage, uint32_t k) {
            const uint32_t base = lds0 + stage * kStage + wave * 1024u;
            const uint32_t outside = k + kl < k1 ? 0u : 0xFFFFFFFFu;
#pragma unroll
            for (int j = 0; j < kLoadsA; ++j) piece_to_lds(base + j * NW * 1024u, (voffA + j * stepA + k * 2u) | outside, ra);
#pragma unroll
            for (int j = 0; j < kLoadsB; ++j) piece_to_lds(base + kABytes + j * NW * 1024u, (voffB + j * stepB + k * 2u) | outside, rb);
        };
        // fragment (ks, t): row 32 t + lane % 32 of the wave's part, piece 2 ks + lane / 32, whose place differs by ks only in bits 5, 6
        const uint32_t rA = wm * WM + (lane & 31u), rB = wn * WN + (lane & 31u), half = lane >> 5;
        uint32_t fA[4], fB[4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const uint32_t place = ((ks * 2u + half) ^ (lane & 7u)) * 16u;
            fA[ks] = rA * 128u + place;
            fB[ks] = kABytes + rB * 128u + place;
        }
        // the compiler must see a store to the array: everything else arrives behind its back
        reinterpret_cast<uint32_t*>(sh + 2 * kStage)[threadIdx.x & 255u] = 0u;
        issue(0, k0);
        uint32_t stage = 0;
        for (uint32_t k = k0; k < k1; k += kStepK) {
            // this wave's pieces of the step have landed and it has what it read of the other stage; then everybody's
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (k + kStepK < k1) issue(stage ^ 1u, k + kStepK);
            const uint8_t* at = sh + stage * kStage;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                bf8v a[MT], b[NT];
#pragma unroll
                for (int t = 0; t < MT; ++t) a[t] = *reinterpret_cast<const bf8v*>(at + fA[ks] + t * 32 * 128);
#pragma unroll
                for (int t = 0; t < NT; ++t) b[t] = *reinterpret_cast<const bf8v*>(at + fB[ks] + t * 32 * 128);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[m], b[n], acc[m][n], 0, 0, 0);
                if (kFine) after(k + ks * 16u + 16u);
            }
            if (!kFine) after(k + kStepK);
            stage ^= 1u;
        }
    }
};

}  // namespace vgc
#endif
