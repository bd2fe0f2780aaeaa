// Matrix products C[m, n] = sum_k a[m, k] b[n, k] with bfloat16 operands and float32 accumulators, for operands whose k lies
// contiguous (RowTile), for operands whose m and n do (ColumnTile) and for one of each (MixedTile).
//
// A workgroup owns a BM x BN tile of C, a wave a WM x WN part of it in 32 x 32 tiles of v_mfma_f32_32x32x16_bf16.  Steps of BK k
// travel from global memory straight into a ring of S stages in LDS (buffer loads with the LDS modifier: lane l of a wave-wide
// load deposits its 16 bytes at M0 + 16 l), S steps ahead of the one being multiplied.
//
// An operand may consist of several planes that add up to it (an exact cut of a float, or a value in two pieces); a product of
// operands is the sum over the pairs of planes that matter, smallest first, formed from the same fragments in one pass: three
// planes a side meet in the six pairs that reach 2^-24, two or three planes meet one in as many.
//
// Lane l of the instruction holds, for row m = l % 32, the eight k = 8 (l / 32) .. + 7.  Its 16 results are
// C[m = 8 (i / 4) + 4 (l / 32) + i % 4][n = l % 32], i = 0..15.
#ifndef VGC_GEMM_H
#define VGC_GEMM_H

#include "vgc_internal.h"

namespace vgc {

typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef short s8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef int i4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s4v* lds_s4v_ptr;

// An operand in memory: element (row, column) of plane q at base[q * plane + row * ld + column].  base, ld and plane are multiples of
// 16 bytes.  What a workgroup addresses of a plane has to span less than 2^32 bytes.
struct Matrix {
    const uint16_t* base;
    uint32_t rows, ld;
    uint64_t plane;
};

// 16 bytes a lane from the bounded buffer `rsrc` (byte offset voff) to LDS byte address lds + 16 * lane.  Lanes outside the range
// deposit zeros.  Counted by vmcnt.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"              // m0 is named as clobbered on purpose
__device__ __forceinline__ void piece_to_lds(uint32_t lds, uint32_t voff, i4v rsrc) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(lds), "v"(voff), "s"(rsrc) : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N> __device__ __forceinline__ void wait_pieces_but() {       // ... and for what this wave has asked of LDS
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(N) : "memory");
}

// Rows [row0, row0 + count) of a plane as a bounded buffer.
__device__ __forceinline__ i4v rows_rsrc(const Matrix& M, int plane, uint32_t row0, uint32_t count) {
    const uint64_t addr = reinterpret_cast<uint64_t>(M.base) + ((uint64_t)plane * M.plane + (uint64_t)row0 * M.ld) * 2u;
    const uint32_t left = row0 < M.rows ? min(M.rows - row0, count) : 0u;
    i4v r;                                                   // uniform values; the asm operand must be scalar registers
    r[0] = (int)__builtin_amdgcn_readfirstlane((uint32_t)addr);
    r[1] = (int)__builtin_amdgcn_readfirstlane((uint32_t)(addr >> 32) & 0xFFFFu);
    r[2] = (int)__builtin_amdgcn_readfirstlane(left * M.ld * 2u);
    r[3] = 0x00020000;
    return r;
}

// Logical number of a workgroup so that each of the eight XCDs, which take workgroups in turn, gets a contiguous range: those
// that share operand rows share an L2.
__device__ __forceinline__ uint32_t xcd_contiguous(uint32_t id, uint32_t total) {
    const uint32_t per = total / 8u, rem = total % 8u, xcd = id % 8u, slot = id / 8u;
    return xcd * per + min(xcd, rem) + slot;
}

// Tile number `id` of tiles_m x tiles_n, in bands of eight columns: the 32 tiles that an XCD's compute units work on at a time are
// four rows of tiles by eight columns and read 12 panels of the operands instead of 18 or more.
struct TilePlace { uint32_t m, n; };
__device__ __forceinline__ TilePlace in_bands(uint32_t id, uint32_t tiles_m, uint32_t tiles_n) {
    const uint32_t band = id / (tiles_m * 8u), rest = id - band * tiles_m * 8u, width = min(8u, tiles_n - band * 8u);
    return TilePlace{rest / width, band * 8u + rest % width};
}

// The pairs of planes of a product, smallest first.
template <int PA, int PB> struct Pairs;
template <> struct Pairs<1, 1> { static constexpr int n = 1, a[1] = {0}, b[1] = {0}; };
template <> struct Pairs<1, 2> { static constexpr int n = 2, a[2] = {0, 0}, b[2] = {1, 0}; };
template <> struct Pairs<2, 1> { static constexpr int n = 2, a[2] = {1, 0}, b[2] = {0, 0}; };
template <> struct Pairs<3, 1> { static constexpr int n = 3, a[3] = {2, 1, 0}, b[3] = {0, 0, 0}; };
template <> struct Pairs<2, 2> { static constexpr int n = 4, a[4] = {1, 1, 0, 0}, b[4] = {1, 0, 1, 0}; };
template <> struct Pairs<3, 3> { static constexpr int n = 6, a[6] = {2, 0, 1, 1, 0, 0}, b[6] = {0, 2, 1, 0, 1, 0}; };

template <int BM_, int BN_, int WM_, int WN_, int BK_, int S_, int PA_, int PB_> struct TileShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, S = S_, PA = PA_, PB = PB_;
    static constexpr int NW = (BM / WM) * (BN / WN), MT = WM / 32, NT = WN / 32, KS = BK / 16;
    static constexpr uint32_t kPlaneA = BM * BK * 2, kPlaneB = BN * BK * 2, kStage = PA * kPlaneA + PB * kPlaneB;
    static constexpr uint32_t kLds = S * kStage + 1024;      // (the last KiB: see loop)
    static constexpr int kPerA = (int)(kPlaneA / 1024) / NW, kPerB = (int)(kPlaneB / 1024) / NW, kPer = PA * kPerA + PB * kPerB;
    static_assert(kPlaneA % (1024 * NW) == 0 && kPlaneB % (1024 * NW) == 0, "every wave issues the same loads");
    static_assert(S >= 2 && (S - 1) * kPer < 64, "vmcnt");
    typedef Pairs<PA, PB> P;

    static __device__ __forceinline__ uint32_t wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    static __device__ __forceinline__ uint32_t wave_m() { return wave() / (BN / WN) * WM; }
    static __device__ __forceinline__ uint32_t wave_n() { return wave() % (BN / WN) * WN; }

    // The loop both kinds share.  issue(stage, step, i): request i of a step; fa/fb(stage, plane, ks, t): a fragment; after(step, ks): acc
    // holds all up to there.
    //
    // A phase is 16 k.  While the instructions of a phase run, the fragments of the next one are read into the other of two
    // register sets.  The workgroup meets once a step, before the last phase: by then every wave has its pieces of the next step in
    // LDS and has received every fragment of the present one, whose stage is free for the request S steps ahead; the next step's
    // first fragments are read in the last phase.  Requests and reads are dealt out between the matrix instructions: eight waves
    // that issue theirs in one go after the barrier wait for each other's, and the matrix pipes for them.
    template <typename Issue, typename FragA, typename FragB, typename After>
    static __device__ __forceinline__ void loop(f16v (&acc)[MT][NT], uint8_t* sh, uint32_t steps, Issue issue, FragA fa, FragB fb, After after) {
        static_assert(KS % 2 == 0, "phases take the two register sets in turn");
        constexpr int kProducts = P::n * NT * MT, kReads = PA * MT + PB * NT;
        // the compiler must see a store to the array: everything else arrives behind its back
        reinterpret_cast<uint32_t*>(sh + S * kStage)[threadIdx.x & 255u] = 0u;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < kPer; ++i) issue((uint32_t)s * kStage, (uint32_t)s, i);
        bf8v a[2][PA][MT], b[2][PB][NT];
        auto read = [&](int set, uint32_t stage, int ks, int i) {          // b's fragments first
            if (i < PB * NT) b[set][i / NT][i % NT] = fb(stage, i / NT, ks, i % NT);
            else a[set][(i - PB * NT) / MT][(i - PB * NT) % MT] = fa(stage, (i - PB * NT) / MT, ks, (i - PB * NT) % MT);
        };
        auto multiply = [&](int set, int j) {
            const int e = j / (NT * MT), n = j / MT % NT, m = j % MT;
            acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[set][P::a[e]][m], b[set][P::b[e]][n], acc[m][n], 0, 0, 0);
        };
        wait_pieces_but<(S - 1) * kPer>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < kReads; ++i) read(0, 0, 0, i);
        uint32_t cur = 0;
        for (uint32_t step = 0; step < steps; ++step) {
            const uint32_t next = cur + kStage == S * kStage ? 0u : cur + kStage;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const bool last = ks == KS - 1;
                if (last) {
                    wait_pieces_but<(S - 2) * kPer>();
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                }
#pragma unroll
                for (int j = 0; j < kProducts; ++j) {
                    multiply(ks & 1, j);
#pragma unroll
                    for (int i = 0; i < kReads; ++i)
                        if (i * kProducts / kReads == j) read((ks + 1) & 1, last ? next : cur, last ? 0 : ks + 1, i);
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        if (last && i * kProducts / kPer == j) issue(cur, step + S, i);      // (past the last step: zeros that nobody reads)
                    __builtin_amdgcn_sched_barrier(0);
                }
                after(step, ks);
            }
            cur = next;
        }
        wait_pieces_but<0>();                                // nothing is on its way into LDS when it is used for something else
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
};

// k contiguous: rows of a are m, of b are n.  A staged row is BK * 2 bytes, pieces of 16; piece q of row r lies at place
// q ^ mask(r).  A read of 16 bytes a lane is served 16 lanes at a time, rows 0..3, 12..15, 20..23, 24..27 of 32 and then the others;
// with the masks below each such sixteen lies in sixteen different groups of four banks (with r % 8 and r / 2 % 4 in their places
// half of the LDS cycles were conflicts).  The exchange is made on the way in by choosing which global piece each lane fetches, and
// on the way out in the fragment addresses.
template <typename Shape> struct RowTile : Shape {
    using Shape::BM; using Shape::BN; using Shape::BK; using Shape::NW; using Shape::PA; using Shape::PB;
    static constexpr uint32_t kRowBytes = BK * 2, kPieces = BK / 8, kRowsPerLoad = 1024 / kRowBytes;
    static __device__ __forceinline__ uint32_t mask(uint32_t row) { return BK == 64 ? ((row >> 1) & 3u) | ((row >> 2) & 4u) : (row >> 3) & 3u; }

    // acc += a[m0 .., k] b[n0 .., k] over k < K (a multiple of 8).  b's rows lie where row_of(n) says (n >= count_n or row_of(n)
    // = ~0: zeros), relative to row b_row0, within b_rows of it.
    template <typename RowOf, typename After>
    static __device__ __forceinline__ void run(f16v (&acc)[Shape::MT][Shape::NT], uint8_t* sh, const Matrix& A, const Matrix& B, uint32_t m0,
                                               uint32_t b_row0, uint32_t b_rows, RowOf row_of, uint32_t K, After after) {
        const uint32_t lane = threadIdx.x & 63u, wave = Shape::wave();
        const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)sh) + wave * 1024u;
        i4v ra[PA], rb[PB];
#pragma unroll
        for (int q = 0; q < PA; ++q) ra[q] = rows_rsrc(A, q, m0, BM);
#pragma unroll
        for (int q = 0; q < PB; ++q) rb[q] = rows_rsrc(B, q, b_row0, b_rows);
        // load j of a wave covers kRowsPerLoad rows from (j NW + wave) kRowsPerLoad on
        const uint32_t row = wave * kRowsPerLoad + lane / kPieces, piece = (lane % kPieces) ^ mask(row);
        static_assert((NW * kRowsPerLoad) % 32 == 0, "the exchange is the same in every load of a lane");
        const uint32_t kl = piece * 8u, offA = (row * A.ld + kl) * 2u, stepA = NW * kRowsPerLoad * A.ld * 2u;
        uint32_t offB[Shape::kPerB], noneB[Shape::kPerB];
#pragma unroll
        for (int j = 0; j < Shape::kPerB; ++j) {
            const uint32_t r = row_of(row + j * NW * kRowsPerLoad);
            noneB[j] = r == 0xFFFFFFFFu ? r : 0u;
            offB[j] = (r * B.ld + kl) * 2u;
        }
        auto issue = [&](uint32_t stage, uint32_t step, int i) {
            const uint32_t k = step * BK, outside = k + kl < K ? 0u : 0xFFFFFFFFu;
            if (i < PA * Shape::kPerA) {
                const int q = i / Shape::kPerA, j = i % Shape::kPerA;
                piece_to_lds(lds0 + stage + q * Shape::kPlaneA + j * NW * 1024u, (offA + j * stepA + k * 2u) | outside, ra[q]);
            } else {
                const int q = (i - PA * Shape::kPerA) / Shape::kPerB, j = (i - PA * Shape::kPerA) % Shape::kPerB;
                piece_to_lds(lds0 + stage + PA * Shape::kPlaneA + q * Shape::kPlaneB + j * NW * 1024u, (offB[j] + k * 2u) | outside | noneB[j], rb[q]);
            }
        };
        // fragment (ks, t): row 32 t + lane % 32 of the wave's part, piece 2 ks + lane / 32
        const uint32_t rA = (Shape::wave_m() + (lane & 31u)) * kRowBytes, rB = (Shape::wave_n() + (lane & 31u)) * kRowBytes;
        uint32_t place[Shape::KS];
#pragma unroll
        for (int ks = 0; ks < Shape::KS; ++ks) place[ks] = ((ks * 2u + (lane >> 5)) ^ mask(lane & 31u)) * 16u;
        auto fa = [&](uint32_t stage, int q, int ks, int t) {
            return *reinterpret_cast<const bf8v*>(sh + stage + q * Shape::kPlaneA + rA + place[ks] + t * 32u * kRowBytes);
        };
        auto fb = [&](uint32_t stage, int q, int ks, int t) {
            return *reinterpret_cast<const bf8v*>(sh + stage + PA * Shape::kPlaneA + q * Shape::kPlaneB + rB + place[ks] + t * 32u * kRowBytes);
        };
        Shape::loop(acc, sh, (K + BK - 1) / BK, issue, fa, fb, after);
    }
};

// m and n contiguous: rows of both operands are k.  Fragments come through the transposing read ds_read_b64_tr_b16: within 16
// lanes, lane r supplies the address of 4 consecutive b16 and lane i receives element i % 4 from the addresses of lanes
// i / 4 + 4 j, j = 0..3; with lane r pointing at row k0 + r / 4, columns m0 + 4 (r % 4) .. + 3, lane i receives k0 .. k0 + 3 of
// column m0 + i.  The 64-byte units of a staged row are exchanged by row % 4, so that rows k0 .. k0 + 3 of one unit start 16 banks
// apart.
template <typename Shape> struct ColumnTile : Shape {
    using Shape::BM; using Shape::BN; using Shape::BK; using Shape::NW; using Shape::PA; using Shape::PB;
    static_assert(BM >= 128 && BN >= 128, "four units a row");

    // acc += a[k, m0 ..] b[k, n0 ..] over rows k in [k0, k1).  Columns past a row's end read its successor's, or zeros.
    // after(step, ks) as for the loop; steps count from k0.
    static __device__ __forceinline__ void run(f16v (&acc)[Shape::MT][Shape::NT], uint8_t* sh, const Matrix& A, const Matrix& B, uint32_t m0,
                                               uint32_t n0, uint32_t k0, uint32_t k1) {
        run(acc, sh, A, B, m0, n0, k0, k1, [](uint32_t, int) {});
    }
    template <typename After>
    static __device__ __forceinline__ void run(f16v (&acc)[Shape::MT][Shape::NT], uint8_t* sh, const Matrix& A, const Matrix& B, uint32_t m0,
                                               uint32_t n0, uint32_t k0, uint32_t k1, After after) {
        const uint32_t lane = threadIdx.x & 63u, wave = Shape::wave();
        const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)sh) + wave * 1024u;
        i4v ra[PA], rb[PB];
#pragma unroll
        for (int q = 0; q < PA; ++q) ra[q] = rows_rsrc(A, q, k0, k1 - k0);
#pragma unroll
        for (int q = 0; q < PB; ++q) rb[q] = rows_rsrc(B, q, k0, k1 - k0);
        constexpr uint32_t nprA = BM / 8, nprB = BN / 8, rpiA = 64 / nprA, rpiB = 64 / nprB;       // pieces a row, rows a load
        auto offset = [&](uint32_t npr, uint32_t rpi, uint32_t ld, uint32_t col0) {
            const uint32_t row = wave * rpi + lane / npr, p = lane % npr, piece = (((p >> 2) ^ (row & 3u)) << 2) | (p & 3u);
            return (row * ld + col0 + piece * 8u) * 2u;
        };
        const uint32_t offA = offset(nprA, rpiA, A.ld, m0), offB = offset(nprB, rpiB, B.ld, n0);
        static_assert((NW * rpiA) % 4 == 0 && (NW * rpiB) % 4 == 0, "the exchange is the same in every load of a lane");
        const uint32_t stepA = NW * rpiA * A.ld * 2u, stepB = NW * rpiB * B.ld * 2u, rowsA = BK * A.ld * 2u, rowsB = BK * B.ld * 2u;
        // (rows past k1 lie past the buffer; steps past the last one may wrap around 2^32, so they are asked for outside)
        const uint32_t steps = (k1 - k0 + BK - 1) / BK;
        auto issue = [&](uint32_t stage, uint32_t step, int i) {
            const uint32_t outside = step < steps ? 0u : 0xFFFFFFFFu;
            if (i < PA * Shape::kPerA) {
                const int q = i / Shape::kPerA, j = i % Shape::kPerA;
                piece_to_lds(lds0 + stage + q * Shape::kPlaneA + j * NW * 1024u, (offA + j * stepA + step * rowsA) | outside, ra[q]);
            } else {
                const int q = (i - PA * Shape::kPerA) / Shape::kPerB, j = (i - PA * Shape::kPerA) % Shape::kPerB;
                piece_to_lds(lds0 + stage + PA * Shape::kPlaneA + q * Shape::kPlaneB + j * NW * 1024u, (offB + j * stepB + step * rowsB) | outside, rb[q]);
            }
        };
        const uint32_t r = lane & 15u, mhalf = (lane >> 4) & 1u, frow = (lane >> 5) * 8u + (r >> 2);
        uint32_t fA[Shape::MT], fB[Shape::NT];
#pragma unroll
        for (int t = 0; t < Shape::MT; ++t) fA[t] = frow * (BM * 2u) + (((Shape::wave_m() / 32u + t) ^ (frow & 3u)) * 64u) + mhalf * 32u + (r & 3u) * 8u;
#pragma unroll
        for (int t = 0; t < Shape::NT; ++t)
            fB[t] = PA * Shape::kPlaneA + frow * (BN * 2u) + (((Shape::wave_n() / 32u + t) ^ (frow & 3u)) * 64u) + mhalf * 32u + (r & 3u) * 8u;
        auto read = [&](const uint8_t* p, uint32_t four_rows) {
            const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v_ptr)(p));
            const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v_ptr)(p + four_rows));
            const s8v v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            return __builtin_bit_cast(bf8v, v);
        };
        auto fa = [&](uint32_t stage, int q, int ks, int t) { return read(sh + stage + q * Shape::kPlaneA + fA[t] + ks * 16 * BM * 2, 4 * BM * 2); };
        auto fb = [&](uint32_t stage, int q, int ks, int t) { return read(sh + stage + q * Shape::kPlaneB + fB[t] + ks * 16 * BN * 2, 4 * BN * 2); };
        Shape::loop(acc, sh, steps, issue, fa, fb, after);
    }
};

// m contiguous in a, whose rows are k, and k contiguous in b, whose rows are n: a's stages lie and are read as ColumnTile's, b's as RowTile's.
template <typename Shape> struct MixedTile : Shape {
    using Shape::BM; using Shape::BN; using Shape::BK; using Shape::NW; using Shape::PA; using Shape::PB;
    typedef RowTile<Shape> Rows;
    static_assert(BM >= 128, "four units a row");

    // acc += a[k, m0 ..] b[n0 .., k] over k < K (a multiple of 8, or beyond it zeros in a's rows and in b).  Columns past a row's end of a read its
    // successor's, or zeros; rows past b's end are zeros.
    template <typename After>
    static __device__ __forceinline__ void run(f16v (&acc)[Shape::MT][Shape::NT], uint8_t* sh, const Matrix& A, const Matrix& B, uint32_t m0,
                                               uint32_t n0, uint32_t K, After after) {
        const uint32_t lane = threadIdx.x & 63u, wave = Shape::wave();
        const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)sh) + wave * 1024u;
        i4v ra[PA], rb[PB];
#pragma unroll
        for (int q = 0; q < PA; ++q) ra[q] = rows_rsrc(A, q, 0, K);
#pragma unroll
        for (int q = 0; q < PB; ++q) rb[q] = rows_rsrc(B, q, n0, BN);
        constexpr uint32_t nprA = BM / 8, rpiA = 64 / nprA;
        static_assert((NW * rpiA) % 4 == 0 && (NW * Rows::kRowsPerLoad) % 32 == 0, "the exchanges are the same in every load of a lane");
        const uint32_t arow = wave * rpiA + lane / nprA, ap = lane % nprA, apiece = (((ap >> 2) ^ (arow & 3u)) << 2) | (ap & 3u);
        const uint32_t offA = (arow * A.ld + m0 + apiece * 8u) * 2u, stepA = NW * rpiA * A.ld * 2u, rowsA = BK * A.ld * 2u;
        const uint32_t brow = wave * Rows::kRowsPerLoad + lane / Rows::kPieces, kl = ((lane % Rows::kPieces) ^ Rows::mask(brow)) * 8u;
        const uint32_t offB = (brow * B.ld + kl) * 2u, stepB = NW * Rows::kRowsPerLoad * B.ld * 2u;
        const uint32_t steps = (K + BK - 1) / BK;
        auto issue = [&](uint32_t stage, uint32_t step, int i) {
            if (i < PA * Shape::kPerA) {
                const int q = i / Shape::kPerA, j = i % Shape::kPerA;
                piece_to_lds(lds0 + stage + q * Shape::kPlaneA + j * NW * 1024u, (offA + j * stepA + step * rowsA) | (step < steps ? 0u : 0xFFFFFFFFu), ra[q]);
            } else {
                const int q = (i - PA * Shape::kPerA) / Shape::kPerB, j = (i - PA * Shape::kPerA) % Shape::kPerB;
                const uint32_t k = step * BK;
                piece_to_lds(lds0 + stage + PA * Shape::kPlaneA + q * Shape::kPlaneB + j * NW * 1024u,
                             (offB + j * stepB + k * 2u) | (k + kl < K ? 0u : 0xFFFFFFFFu), rb[q]);
            }
        };
        const uint32_t r = lane & 15u, mhalf = (lane >> 4) & 1u, frow = (lane >> 5) * 8u + (r >> 2);
        uint32_t fA[Shape::MT], place[Shape::KS];
#pragma unroll
        for (int t = 0; t < Shape::MT; ++t) fA[t] = frow * (BM * 2u) + (((Shape::wave_m() / 32u + t) ^ (frow & 3u)) * 64u) + mhalf * 32u + (r & 3u) * 8u;
        const uint32_t rB = (Shape::wave_n() + (lane & 31u)) * Rows::kRowBytes;
#pragma unroll
        for (int ks = 0; ks < Shape::KS; ++ks) place[ks] = ((ks * 2u + (lane >> 5)) ^ Rows::mask(lane & 31u)) * 16u;
        auto fa = [&](uint32_t stage, int q, int ks, int t) {
            const uint8_t* p = sh + stage + q * Shape::kPlaneA + fA[t] + ks * 16 * BM * 2;
            const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v_ptr)(p));
            const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v_ptr)(p + 4 * BM * 2));
            const s8v v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            return __builtin_bit_cast(bf8v, v);
        };
        auto fb = [&](uint32_t stage, int q, int ks, int t) {
            return *reinterpret_cast<const bf8v*>(sh + stage + PA * Shape::kPlaneA + q * Shape::kPlaneB + rB + place[ks] + t * 32u * Rows::kRowBytes);
        };
        Shape::loop(acc, sh, steps, issue, fa, fb, after);
    }
};

// Products far below the sum that a matrix instruction adds them to come out too small rather than rounded: with the six products of
// planes that float32 operands bring for every 16 k, sums shrink as they grow (bfloat16 operands, whose products are of one
// size, show none of it).  Taken out of the instructions' reach every kPart k, a sum is rounded as float sums are.  0: left there.
template <typename Shape, uint32_t kPart> struct InParts {
    f16v total[Shape::MT][Shape::NT] = {};
    __device__ __forceinline__ void after(f16v (&acc)[Shape::MT][Shape::NT], uint32_t step, int ks) {
        if (ks != Shape::KS - 1 || (step + 1u) * Shape::BK % kPart != 0u) return;
#pragma unroll
        for (int m = 0; m < Shape::MT; ++m)
#pragma unroll
            for (int n = 0; n < Shape::NT; ++n) { total[m][n] += acc[m][n]; acc[m][n] = f16v{}; }
    }
    __device__ __forceinline__ void end(f16v (&acc)[Shape::MT][Shape::NT]) {
#pragma unroll
        for (int m = 0; m < Shape::MT; ++m)
#pragma unroll
            for (int n = 0; n < Shape::NT; ++n) acc[m][n] += total[m][n];
    }
};
template <typename Shape> struct InParts<Shape, 0u> {
    __device__ __forceinline__ void after(f16v (&)[Shape::MT][Shape::NT], uint32_t, int) {}
    __device__ __forceinline__ void end(f16v (&)[Shape::MT][Shape::NT]) {}
};

}  // namespace vgc
#endif
