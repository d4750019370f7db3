// The 4-bit format of a paged cache: 16 elements share a scale S = 16 e, e of type e5m2, and are held as n = x / S in -7 .. 7.
//
// e has three significant bits, so that n * S is exact in 16-bit floats of either kind, and so are the multiples of e with which the
// attention turns codes into numbers (paged_attn_q4.cu); a byte of it is the upper half of an fp16.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "sm100.cuh"

namespace metok {

#ifdef __CUDACC__
constexpr float kQ4Unit = 16.f, kQ4Most = 56.f;        // S = kQ4Unit * e, e at most kQ4Most
constexpr uint32_t kQ4NaN = 0x7Fu;                     // the scale of a block with a NaN or an infinity

// Sixteen elements, as they lie in memory, to fp32.
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
__device__ __forceinline__ float max_nan(float a, float b) {            // a NaN stays one
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The smallest e of its type with top <= 7.5 * 16 * e, but at most kQ4Most.
__device__ __forceinline__ float q4_scale(float top) {
    if (top < 120.f * 6.103515625e-5f) {               // few blocks: below 2^-14 the numbers of the type are 2^-16 apart
        const float e = ceilf(top * (65536.f / 120.f)) * 1.52587890625e-5f, lower = e - 1.52587890625e-5f;
        if (top > 120.f * e) return e + 1.52587890625e-5f;               // (the product was rounded; 120 e is exact)
        return lower >= 0.f && top <= 120.f * lower ? lower : e;
    }
    // a quotient that is a little too small, up to three bits: e, or the number before it
    const uint32_t below = (__float_as_uint(top * (0.99999905f / 120.f)) + 0x1FFFFFu) & ~0x1FFFFFu;
    return fminf(__uint_as_float(top > 120.f * __uint_as_float(below) ? below + 0x200000u : below), kQ4Most);
}

// Holds sixteen elements: their codes (element d in nibble d % 8 of code[d / 8]); returns the scale's byte.
//
// n = x / S rounded to even has to be right where x lies halfway between two multiples of S, which bf16 elements often do, and 1 / S is no
// number of fp32.  A quotient q corrected by its remainder, q + (x - q S) / S, is off by next to nothing before its last rounding, as the
// remainder is exact: so it is c + 1/2 where that is the quotient, and nowhere else, since with three bits in S other quotients are more than half a
// step of fp32 away from it.  The codes of four elements are added up in fp32: sums of n 16^j, exact.
__device__ __forceinline__ uint32_t q4_hold(float (&x)[16], uint32_t (&code)[2]) {
    using namespace sm100;
    float top = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) top = max_nan(top, fabsf(x[i]));
    const float e = q4_scale(top), S = kQ4Unit * e;
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(S));
    if (!(top < 7.46f * S)) {                          // few blocks: zeros, what would round to 8 or is beyond the largest scale, no numbers
        if (!(top <= 3.402823466e38f) || top == 0.f) {
            code[0] = code[1] = 0x88888888u;
            return top == 0.f ? 0u : kQ4NaN;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = fminf(fmaxf(x[i], -7.f * S), 7.f * S);
    }
    const uint64_t inv2 = pair(inv, inv), neg2 = pair(-S, -S), magic = pair(12582912.f, 12582912.f), unmagic = pair(-12582912.f, -12582912.f),
                   next = pair(256.f, 256.f);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint64_t n[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint64_t v = pair(x[8 * w + 2 * j], x[8 * w + 2 * j + 1]), q = mul_pair(v, inv2);
            n[j] = add_pair(add_pair(fma_pair(fma_pair(q, neg2, v), inv2, q), magic), unmagic);
        }
        float half[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float even, odd;
            unpair(fma_pair(n[2 * j + 1], next, n[2 * j]), even, odd);
            half[j] = fmaf(odd, 16.f, even) + (12582912.f + 34952.f);    // 8 for every nibble: 0x8888
        }
        code[w] = __byte_perm(__float_as_uint(half[0]), __float_as_uint(half[1]), 0x5410);
    }
    return (uint32_t)__half_as_ushort(__float2half_rn(e)) >> 8;
}

// What the eight elements of a word stand for, as they lie in memory.  A nibble c is masked into the fraction of a bf16 number, 128 + c, and
// one multiply-add gives (128 + c) S - 136 S: of seven bits and exact, as S has three.
template <typename T>
__device__ __forceinline__ void q4_stands_for(uint32_t c, uint32_t scale, uint4 (&v)[sizeof(T) / 2]) {
    const float S = kQ4Unit * __half2float(__ushort_as_half((unsigned short)(scale << 8)));
    const __nv_bfloat162 s2 = __float2bfloat162_rn(S), off = __float2bfloat162_rn(-136.f * S);
    uint32_t p[4];                                     // elements j and j + 4
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t m;
        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(m) : "r"(c >> (4 * j)), "r"(0x000F000Fu), "r"(0x43004300u));
        const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&m), s2, off);
        p[j] = *reinterpret_cast<const uint32_t*>(&r);
    }
    const uint32_t w[4] = {__byte_perm(p[0], p[1], 0x5410), __byte_perm(p[2], p[3], 0x5410), __byte_perm(p[0], p[1], 0x7632),
                           __byte_perm(p[2], p[3], 0x7632)};             // elements 2 i, 2 i + 1
    if constexpr (sizeof(T) == 2) {
        v[0] = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = make_uint4(w[2 * i] << 16, w[2 * i] & 0xFFFF0000u, w[2 * i + 1] << 16, w[2 * i + 1] & 0xFFFF0000u);
    }
}
#endif

}  // namespace metok
