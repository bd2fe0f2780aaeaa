// Rows of activations in pieces of eight elements, shared by the kernels that go through such rows, and the 8-bit form of a block of them, by
// those of vgc_act8.hip and vgc_norm.hip.
#ifndef VGC_ROWS_H
#define VGC_ROWS_H

#include "vgc_internal.h"

namespace vgc {

// A lane's eight consecutive elements of a row, widened to float.  Rows begin at any multiple of the element's size (a row of
// odd length moves the next one), which one load of 16 bytes takes on this target.  n: elements of the piece that exist (8 or more:
// all, 0 or less: none).  The last piece of a row may be short.  It is written element by element; reading it so makes the wave wait for
// what it asked for before (rows of 1023 bfloat16: backward 193 us, of 1024: 102), so where eight elements are there to be read all the
// same (rows follow: at_end false) they are read, and clipped when they are used.
typedef uint32_t any_u4 __attribute__((ext_vector_type(4), aligned(2)));
typedef float any_f4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t any_u2 __attribute__((ext_vector_type(2), aligned(1)));

template <typename T> struct Raw8;                           // as it is in memory: the loads of a later row are kept like this
template <> struct Raw8<uint16_t> { uint32_t w[4]; };
template <> struct Raw8<float> { float f[8]; };

__device__ __forceinline__ Raw8<uint16_t> load8(const uint16_t* p, int n, bool at_end = true) {
    Raw8<uint16_t> r = {};
    if (n >= 8 || (n > 0 && !at_end)) {
        const any_u4 v = *reinterpret_cast<const any_u4*>(p);
        for (int i = 0; i < 4; ++i) r.w[i] = v[i];
    }
    if (__builtin_expect(n > 0 && n < 8 && at_end, 0)) {     // (a branch of its own: lanes without a piece do not enter it)
        for (int i = 0; i < 7; ++i)
            if (i < n) r.w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    }
    return r;
}
__device__ __forceinline__ Raw8<float> load8(const float* p, int n, bool at_end = true) {
    Raw8<float> r = {};
    if (n >= 8 || (n > 0 && !at_end)) {
        const any_f4 a = *reinterpret_cast<const any_f4*>(p), b = *reinterpret_cast<const any_f4*>(p + 4);
        for (int i = 0; i < 4; ++i) { r.f[i] = a[i]; r.f[4 + i] = b[i]; }
    }
    if (__builtin_expect(n > 0 && n < 8 && at_end, 0)) {
        for (int i = 0; i < 7; ++i)
            if (i < n) r.f[i] = p[i];
    }
    return r;
}
__device__ __forceinline__ void clip8(Raw8<uint16_t>& r, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] &= n >= 2 * i + 2 ? 0xFFFFFFFFu : n == 2 * i + 1 ? 0xFFFFu : 0u;
}
__device__ __forceinline__ void clip8(Raw8<float>& r, int n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.f[i] = i < n ? r.f[i] : 0.f;
}
// Whether eight elements from a place of this row may reach past the rows' array: not where at least eight rows follow.
__device__ __forceinline__ bool rows_at_end(uint64_t row, uint64_t R) { return row + 8u >= R; }
__device__ __forceinline__ void widen8(const Raw8<uint16_t>& r, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(r.w[i] << 16); f[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void widen8(const Raw8<float>& r, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = r.f[i];
}

// Two floats rounded to the nearest bfloat16, ties to even, the first in the low half; a NaN stays one.
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    const bf2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&f)[8], int n) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = two_bf16(f[2 * i], f[2 * i + 1]);
    if (n >= 8) {
        any_u4 v;
        for (int i = 0; i < 4; ++i) v[i] = w[i];
        *reinterpret_cast<any_u4*>(p) = v;
    } else {
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8], int n) {
    if (n >= 8) {
        any_f4 a, b;
        for (int i = 0; i < 4; ++i) { a[i] = f[i]; b[i] = f[4 + i]; }
        *reinterpret_cast<any_f4*>(p) = a;
        *reinterpret_cast<any_f4*>(p + 4) = b;
    } else {
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = f[i];
    }
}
// Results of whole aligned pieces are stored past the caches where what a call touches (bytes) is more than they hold: that leaves room for what is read (the
// linear layer's 16384 x 2048 x 8192 bfloat16 with z 512 -> 477 us).
typedef uint32_t whole_u4 __attribute__((ext_vector_type(4)));
typedef float whole_f4 __attribute__((ext_vector_type(4)));
inline bool past_caches(const void* p, uint32_t row, uint64_t bytes) { return row % 8u == 0u && (reinterpret_cast<uintptr_t>(p) & 15u) == 0u && bytes > (256ull << 20); }
__device__ __forceinline__ void store8_to(uint16_t* p, const float (&f)[8], int n, bool past) {
    if (!past) { store8(p, f, n); return; }
    whole_u4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = two_bf16(f[2 * i], f[2 * i + 1]);
    __builtin_nontemporal_store(v, reinterpret_cast<whole_u4*>(p));
}
__device__ __forceinline__ void store8_to(float* p, const float (&f)[8], int n, bool past) {
    if (!past) { store8(p, f, n); return; }
    const whole_f4 a = {f[0], f[1], f[2], f[3]}, b = {f[4], f[5], f[6], f[7]};
    __builtin_nontemporal_store(a, reinterpret_cast<whole_f4*>(p));
    __builtin_nontemporal_store(b, reinterpret_cast<whole_f4*>(p + 4));
}
__device__ __forceinline__ any_u2 load_codes(const int8_t* p, int n, bool at_end = true) {
    any_u2 v = {0u, 0u};
    if (n >= 8 || (n > 0 && !at_end)) v = *reinterpret_cast<const any_u2*>(p);
    if (__builtin_expect(n > 0 && n < 8 && at_end, 0)) {
        for (int i = 0; i < 7; ++i)
            if (i < n) v[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
    }
    return v;
}
__device__ __forceinline__ void clip_codes(any_u2& v, int n) {
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] &= n >= 4 * i + 4 ? 0xFFFFFFFFu : n <= 4 * i ? 0u : (1u << (8 * (n - 4 * i))) - 1u;
}
__device__ __forceinline__ void store_codes(int8_t* p, any_u2 v, int n) {
    if (n >= 8) {
        *reinterpret_cast<any_u2*>(p) = v;
    } else {
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = (int8_t)(v[i >> 2] >> (8 * (i & 3)));
    }
}

// ---- 8-bit form: a block of up to 32 consecutive elements of a row, codes -127..127, value = code * 2^(field - 127) ----
constexpr uint32_t kAct8Block = 32;
constexpr uint32_t kAct8Lanes = 4;                           // lanes that hold a block between them, eight elements each

// The field of a block whose largest magnitude has the bits `top` (of |x|, compared as integers, so that a NaN is above all):
// the smallest unit 2^(field - 127) of which that magnitude rounds to at most 127, i.e. is below 127.5.  A magnitude in
// [2^k, 2^(k+1)) is 64 to 128 units of 2^(k-6); from 127.5 of them on (mantissa 0x7F0000) the unit is twice that.  Units end
// at 2^-126, so that every value is a normal number or zero, and at 2^121, so that every value is finite: what is above 127 of
// those counts as 127.  A block of zeros, for which any unit would do, has that of
// magnitudes in [1/2, 1).  255: the block holds an infinity or a NaN.
__device__ __forceinline__ uint32_t act8_field(uint32_t top) {
    if (top >= 0x7F800000u) return 255u;
    if (top == 0u) return 120u;
    return (uint32_t)min(max((int)(top >> 23) - 6 + (int)((top & 0x7FFFFFu) >= 0x7F0000u), 1), 248);
}
__device__ __forceinline__ uint32_t act8_top(const float (&f)[8]) {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    return t;
}
__device__ __forceinline__ uint32_t four_lanes_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));      // lanes 1 apart
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));   // 2 apart
}
// Eight codes of a block with this field, rounded to nearest, ties to even (field 255: the codes are 0).  Adding 1.5 2^23 rounds a
// value of at most 2^22 to a whole number and leaves its low byte, in two's complement, in the float's; only the largest unit has to be cut off at 127.
__device__ __forceinline__ any_u2 act8_codes(const float (&f)[8], uint32_t field) {
    const float inverse = __uint_as_float((254u - min(field, 253u)) << 23);
    any_u2 v = {0u, 0u};
    if (field >= 248u) {
        if (field == 255u) return v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i >> 2] |= ((uint32_t)min(max((int)__builtin_rintf(f[i] * inverse), -127), 127) & 0xFFu) << (8 * (i & 3));
        return v;
    }
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __float_as_uint(__builtin_fmaf(f[i], inverse, 12582912.f));
#pragma unroll
    for (int i = 0; i < 2; ++i) {                            // bytes 0 of four words
        const uint32_t lo = __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0C0C0400u), hi = __builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x04000C0Cu);
        v[i] = lo | hi;
    }
    return v;
}
__device__ __forceinline__ void act8_values(any_u2 v, uint32_t field, float (&f)[8]) {
    const float unit = field == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(field << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)(int8_t)(v[i >> 2] >> (8 * (i & 3))) * unit;
}

// Sum over a wave's lanes in a fixed order, the same in every lane.
__device__ __forceinline__ float wave_sum(float x) {
#define VGC_DPP_ADD(ctrl, rows) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, rows, 0xF, false))
    VGC_DPP_ADD(0x111, 0xF);
    VGC_DPP_ADD(0x112, 0xF);
    VGC_DPP_ADD(0x114, 0xF);
    VGC_DPP_ADD(0x118, 0xF);
    VGC_DPP_ADD(0x142, 0xA);
    VGC_DPP_ADD(0x143, 0xC);
#undef VGC_DPP_ADD
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// The same over groups of kL lanes (8, 16, 32 or 64), in each of them.
template <int kL> __device__ __forceinline__ float lanes_sum(float x) {
    if constexpr (kL == 64) return wave_sum(x);
#define VGC_DPP_ADD(ctrl) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xF, 0xF, false))
    VGC_DPP_ADD(0xB1);                                       // lanes 1 apart
    VGC_DPP_ADD(0x4E);                                       // 2 apart
    VGC_DPP_ADD(0x141);                                      // the other four of eight
    if constexpr (kL >= 16) VGC_DPP_ADD(0x140);              // the other eight of a row
#undef VGC_DPP_ADD
    if constexpr (kL >= 32) x += __shfl_xor(x, 16);
    return x;
}

// The largest over groups of 16, 32 or 64 lanes, in each of them (a NaN does not count).
template <int kL> __device__ __forceinline__ void lanes_max(float& x) {
#define VGC_DPP_MAX(ctrl) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xF, 0xF, false)))
    VGC_DPP_MAX(0xB1);
    VGC_DPP_MAX(0x4E);
    VGC_DPP_MAX(0x141);
    VGC_DPP_MAX(0x140);
#undef VGC_DPP_MAX
    if constexpr (kL >= 32) x = fmaxf(x, __shfl_xor(x, 16));
    if constexpr (kL >= 64) x = fmaxf(x, __shfl_xor(x, 32));
}

}  // namespace vgc
#endif
