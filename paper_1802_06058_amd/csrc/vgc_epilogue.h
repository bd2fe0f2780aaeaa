// What follows a product or a norm, eight consecutive elements of a row at a time: activations with their slopes, and dropout whose
// mask is drawn again from a counter wherever it is needed.
#ifndef VGC_EPILOGUE_H
#define VGC_EPILOGUE_H

#include "vgc_rows.h"

namespace vgc {

// ---- activations ------------------------------------------------------------------------------------------------------------
// relu  max(z, 0), slope [z > 0] (0 at a NaN, which stays one in the value);   silu  z s with s = 1 / (1 + e^-z), slope s (1 + z (1 - s))
// gelu  z Phi(z), slope Phi(z) + z phi(z), Phi and phi the normal distribution's share below z and density
//
// Phi(-a) = e^(-a^2 / 2) E(a) for a >= 0, and E, which falls like 1 / a, is t times a polynomial in t = 1 / (1 + 0.35 a): of degree 8, its
// coefficients fitted to E on 0 <= a <= 14 so that the largest relative error is least (3.3e-8; 3.3e-7 evaluated in float32).  Small values
// of Phi so keep their digits, which 1 + erf does not, and the exponential serves the slope too.
// One polynomial for both types: a shorter one within 3.2e-5 for values that are rounded to bfloat16 next took 14 us of 523 less (16384 x 2048 to 8192 with
// z kept), but gave some of them the neighbour of the nearest bfloat16, 1.1e-4 off the nearest ones in the root mean square.
struct Normal { float below, density; };                     // Phi(z), sqrt(2 pi) phi(z)
__device__ __forceinline__ Normal normal_at(float z) {
    const float a = fabsf(z), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, a, 1.f));
    const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);          // (log2(e) / 2)
    float p = -0.0291574303f;
    p = __builtin_fmaf(p, t, 0.144028597f);
    p = __builtin_fmaf(p, t, -0.255833956f);
    p = __builtin_fmaf(p, t, 0.159313608f);
    p = __builtin_fmaf(p, t, -0.0232079124f);
    p = __builtin_fmaf(p, t, 0.105550503f);
    p = __builtin_fmaf(p, t, 0.119821828f);
    p = __builtin_fmaf(p, t, 0.139863436f);
    p = __builtin_fmaf(p, t, 0.139621312f);
    const float q = p * t * e;
    return Normal{z > 0.f ? 1.f - q : q, e};
}
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }

__device__ __forceinline__ void apply_act(int act, float (&f)[8]) {        // (act is uniform)
    if (act == VGC_ACT_RELU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = f[k] < 0.f ? 0.f : f[k];
    } else if (act == VGC_ACT_GELU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] *= normal_at(f[k]).below;
    } else if (act == VGC_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] *= sigmoid(f[k]);
    }
}
// d *= the slope at z.
__device__ __forceinline__ void apply_slope(int act, const float (&z)[8], float (&d)[8]) {
    if (act == VGC_ACT_RELU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) d[k] = z[k] > 0.f ? d[k] : 0.f;
    } else if (act == VGC_ACT_GELU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const Normal n = normal_at(z[k]);
            d[k] *= __builtin_fmaf(z[k] * 0.39894228f, n.density, n.below);
        }
    } else if (act == VGC_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float s = sigmoid(z[k]);
            d[k] *= __builtin_fmaf(s * z[k], 1.f - s, s);
        }
    }
}

// ---- dropout ----------------------------------------------------------------------------------------------------------------
// The generator is Philox with four words and ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC
// 2011): a bijection of the 128-bit counter (piece of eight columns, row, number of the call) under a 64-bit key, of which a round is
// two 32 x 32 bit products.  Its four words are the 16-bit numbers of the piece's eight elements, low halves first; an element whose number
// is below t = round(65536 p) is dropped, the others are multiplied by 65536 / (65536 - t).
// 16 bits an element, so that one bijection serves eight: ten rounds are about 120 issue slots a lane, 15 an element, below what
// the element's bytes take from memory; p is exact to 2^-17 and the mean is kept exactly for the p that is meant.
struct Dropout {
    const uint64_t* rng;      // DEVICE: key, number of the call; read where the kernel runs, so that a recorded launch draws anew when they change
    uint32_t t;               // 0: nothing is dropped (rng is not read), 65536: everything
    float scale;
};
inline Dropout dropout_of(float p, const uint64_t* rng) {
    const uint32_t t = (uint32_t)((double)p * 65536.0 + 0.5);
    return Dropout{rng, t, t < 65536u ? 65536.f / (float)(65536u - t) : 0.f};
}
struct DropoutKey { uint64_t key, call; };
__device__ __forceinline__ DropoutKey dropout_key(const Dropout& D) {
    DropoutKey k = {0, 0};
    if (D.t != 0u && D.t < 65536u) { k.key = D.rng[0]; k.call = D.rng[1]; }
    return k;
}
struct Words4 { uint32_t w[4]; };
__device__ __forceinline__ Words4 philox(uint32_t piece, uint32_t row, const DropoutKey& K) {
    uint32_t c0 = piece, c1 = row, c2 = (uint32_t)K.call, c3 = (uint32_t)(K.call >> 32), k0 = (uint32_t)K.key, k1 = (uint32_t)(K.key >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words4{{c0, c1, c2, c3}};
}
__device__ __forceinline__ void apply_dropout(const Dropout& D, const DropoutKey& K, uint32_t row, uint32_t piece, float (&f)[8]) {
    if (D.t == 0u) return;
    if (D.t >= 65536u) {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = 0.f;
        return;
    }
    const Words4 r = philox(piece, row, K);
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = ((r.w[k >> 1] >> (16 * (k & 1))) & 0xFFFFu) >= D.t ? f[k] * D.scale : 0.f;
}

}  // namespace vgc
#endif
