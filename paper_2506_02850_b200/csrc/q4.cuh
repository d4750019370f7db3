// The 4-bit format of a paged cache: 16 elements share a scale S = 16 e, e of type e5m2, and are held as n = x / S in -7 .. 7.
//
// e has three significant bits, so that n * S is exact in 16-bit floats of either kind, and so are the multiples of e with which the
// attention turns codes into numbers (paged_attn_q4.cu); a byte of it is the upper half of an fp16.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace metok {

#ifdef __CUDACC__
constexpr float kQ4Unit = 16.f, kQ4Most = 56.f;        // S = kQ4Unit * e, e at most kQ4Most
constexpr uint32_t kQ4NaN = 0x7Fu;                     // the scale of a block with a NaN or an infinity

// Sixteen elements, as they lie in memory, to fp32 and back.
template <typename T>
__device__ __forceinline__ void q4_widen(const uint4 (&v)[sizeof(T)], float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) {
                x[4 * i + j] = __uint_as_float(w[j]);
            } else {
                x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
                x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
            }
        }
    }
}
template <typename T>
__device__ __forceinline__ void q4_narrow(const float (&x)[16], uint4 (&v)[sizeof(T)]) {
    uint32_t w[4 * sizeof(T)];
#pragma unroll
    for (int i = 0; i < 4 * (int)sizeof(T); ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
        else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
    }
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) v[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}

// Holds sixteen elements: their codes (element d in nibble d % 8 of code[d / 8]); returns the scale's byte.
__device__ __forceinline__ uint32_t q4_hold(const float (&x)[16], uint32_t (&code)[2]) {
    float top = 0.f;
    bool sound = true;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        top = fmaxf(top, fabsf(x[i]));
        sound &= fabsf(x[i]) <= 3.402823466e38f;
    }
    // The smallest e with top <= 7.5 * 16 * e: the quotient, correctly rounded, never reaches a number of three bits from above (its
    // distance from one is half a step of fp32 at least), then rounded up to the next such number; below 2^-14 these are 2^-16 apart.
    const float want = __fdiv_rn(top, 7.5f * kQ4Unit);
    float e = __uint_as_float((__float_as_uint(want) + 0x1FFFFFu) & ~0x1FFFFFu);
    if (want < 6.103515625e-5f) e = ceilf(want * 65536.f) * 1.52587890625e-5f;
    e = fminf(e, kQ4Most);
    const float S = kQ4Unit * e;
    code[0] = code[1] = 0x88888888u;
    if (!sound) return kQ4NaN;
    if (S > 0.f) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            uint32_t c = 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = fminf(fmaxf(rintf(__fdiv_rn(x[8 * w + j], S)), -7.f), 7.f);
                c |= (uint32_t)((int)n + 8) << (4 * j);
            }
            code[w] = c;
        }
    }
    return (uint32_t)__half_as_ushort(__float2half_rn(e)) >> 8;
}

// What sixteen elements stand for.
__device__ __forceinline__ void q4_stands_for(uint2 code, uint32_t scale, float (&x)[16]) {
    const float S = kQ4Unit * __half2float(__ushort_as_half((unsigned short)(scale << 8)));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = (float)((int)(code.x >> (4 * j) & 15u) - 8) * S;
        x[8 + j] = (float)((int)(code.y >> (4 * j) & 15u) - 8) * S;
    }
}
#endif

}  // namespace metok
