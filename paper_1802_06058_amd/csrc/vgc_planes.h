// Values as bfloat16 planes that add up to them: what the products of vgc_gemm.h are formed from where a value has more digits than one.
#ifndef VGC_PLANES_H
#define VGC_PLANES_H

#include "vgc_rows.h"

namespace vgc {

// The next plane of two floats, the first in the low half, taken out of them: rounded to the nearest bfloat16, so that what is left is
// exact and of either sign.  Three planes of a float32 are all of it (8 bits each, but for bits below the smallest subnormal); planes that were
// cut off instead would leave products too small, all of them, by what the pairs of planes that are not formed hold (logits of 16
// 7e-7 too small).  bfloat16 inputs: two planes are within 2^-18 of an entry of D, three are all of it.
// Of a float32, what would be rounded up to infinity is cut off, and an infinity or a NaN leaves nothing.
template <bool kF32> __device__ __forceinline__ uint32_t next_plane(float& d0, float& d1) {
    uint32_t x = two_bf16(d0, d1);
    if (kF32) {
        const bool finite0 = __builtin_isfinite(d0), finite1 = __builtin_isfinite(d1);
        if (finite0 && (x & 0x7FFFu) == 0x7F80u) x -= 1u;
        if (finite1 && (x & 0x7FFF0000u) == 0x7F800000u) x -= 0x10000u;
        d0 = finite0 ? d0 - __uint_as_float(x << 16) : 0.f;
        d1 = finite1 ? d1 - __uint_as_float(x & 0xFFFF0000u) : 0.f;
        return x;
    }
    d0 -= __uint_as_float(x << 16);
    d1 -= __uint_as_float(x & 0xFFFF0000u);
    return x;
}

// Eight values (used up) as the planes of an operand, 16 bytes each.
template <typename T> __device__ __forceinline__ void store_planes(uint16_t* out, uint64_t plane, float (&f)[8]) {
    if (sizeof(T) == 2) { store8(out, f, 8); return; }
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        any_u4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = next_plane<true>(f[2 * e], f[2 * e + 1]);
        *reinterpret_cast<any_u4*>(out + q * plane) = v;
    }
}

}  // namespace vgc
#endif
