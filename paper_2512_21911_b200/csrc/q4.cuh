// The 4-bit cache: how 64 tokens of a KV head are held, coded and decoded.
//
// A group of 64 values x of a row has a scale D and an offset M in bfloat16, D = (max - min) / 15 * 16 and M = min - D, and a code of four
// bits a value, the nearest to (x - M) / D * 16 - 16.  It stands for bfloat16((1 + c / 16) D + M): 1 + c / 16 is the bfloat16 with the code in
// the bits 3 to 6 of its mantissa, so that two values of a word are a shift, an and-or and a fused product and sum of pairs.  That the
// offset is rounded moves all 16 values of a group by up to 0.05 of their distance, which the codes are chosen for.
//
// A slab of 9216 bytes: codes of the keys [4 chunks of 32 dims][64 tokens][16 bytes], codes of the values [2 chunks of 32 tokens][128 dims]
// [16 bytes], scales of the keys [64 tokens][2 groups][D, M], scales of the values [2 groups][D, M][64 tokens].  A thread that holds a
// token's keys, or a dim's values, reads 16 bytes next to its neighbour's.  A 32-bit word holds eight codes: 2 j in bits 4 j .. 4 j + 3,
// 2 j + 1 sixteen bits higher.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "sv.h"

namespace svq {

constexpr int kSlabTokens = 64, kSlabBytes = SV_Q4_SLAB_BYTES;
constexpr int kOffV = 4096, kOffKScale = 8192, kOffVScale = 8704;

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// 1 + c / 16 of codes 2 j and 2 j + 1 of a word
template <int j>
__device__ __forceinline__ uint32_t steps(uint32_t w)
{
    const uint32_t x = j == 0 ? w << 3 : w >> (4 * j - 3);
    uint32_t d;
    asm("lop3.b32 %0, %1, 0x00780078, %2, 0xEA;" : "=r"(d) : "r"(x), "r"(0x3f803f80u));   // (x & mask) | one, in one instruction
    return d;
}
// ... of the pair that a turn to the right brings to bits 3 and 19 (29: pair 0, 33: pair 1, ...)
__device__ __forceinline__ uint32_t steps_at(uint32_t w, uint32_t turn)
{
    uint32_t d;
    asm("lop3.b32 %0, %1, 0x00780078, %2, 0xEA;" : "=r"(d) : "r"(__funnelshift_r(w, w, turn)), "r"(0x3f803f80u));
    return d;
}
// the eight values of a word, pairs; D and M as pairs
__device__ __forceinline__ void decode(uint32_t w, uint32_t d, uint32_t m, uint32_t *out)
{
    out[0] = fma_bf16x2(steps<0>(w), d, m);
    out[1] = fma_bf16x2(steps<1>(w), d, m);
    out[2] = fma_bf16x2(steps<2>(w), d, m);
    out[3] = fma_bf16x2(steps<3>(w), d, m);
}
__device__ __forceinline__ uint32_t both_low(uint32_t w) { return __byte_perm(w, w, 0x1010); }
__device__ __forceinline__ uint32_t both_high(uint32_t w) { return __byte_perm(w, w, 0x3232); }

// Plain fp32 arithmetic, whatever the compiler is told about division and small numbers.
__device__ __forceinline__ float sub_rn(float a, float b)
{
    float d;
    asm("sub.rn.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float mul_rn(float a, float b)
{
    float d;
    asm("mul.rn.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float div_rn(float a, float b)
{
    float d;
    asm("div.rn.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

__device__ __forceinline__ float lesser(float a, float b)
{
    float d;
    asm("min.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float greater(float a, float b)
{
    float d;
    asm("max.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

struct Scale {
    __nv_bfloat16 d, m;
};
// of a group whose smallest and largest value these are
__device__ __forceinline__ Scale scale_of(float low, float high)
{
    Scale s;
    s.d = __float2bfloat16_rn(mul_rn(div_rn(sub_rn(high, low), 15.f), 16.f));
    s.m = __float2bfloat16_rn(sub_rn(low, __bfloat162float(s.d)));
    return s;
}
// A group without a spread (and one with a NaN or an infinite value, whose scale is none) has the code 0.
__device__ __forceinline__ uint32_t code_of(float x, float d, float m)
{
    if (__float_as_uint(d) - 1u >= 0x7f800000u) return 0;   // (0, or a NaN)
    const float c = rintf(sub_rn(mul_rn(div_rn(sub_rn(x, m), d), 16.f), 16.f));
    return (uint32_t)fminf(fmaxf(c, 0.f), 15.f);
}
// The codes of eight values, value e in nibble e / 2 of the lower (even) or upper half of a word.  One division for the eight: a product with
// 16 / D is off by less than 2^-17, so that what it rounds to is the code wherever it is further than that from the middle between two;
// the others, and scales near the ends of the exponents, take the divisions.  (A number of 2^23 and half as many more has no fraction: adding it rounds.)
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], float d, float m)
{
    const float kRound = 12582912.f;
    uint32_t word = 0;
    float worst = 0.f;
    const bool plain = d >= 0x1p-100f && d <= 0x1p100f;
    const float by = plain ? div_rn(16.f, d) : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = sub_rn(v[e], m), up = fmaf(t, by, kRound - 16.f);
        worst = fmaxf(worst, fabsf(fmaf(t, by, -16.f) - (up - kRound)));
        word |= (__float_as_uint(fminf(fmaxf(up, kRound), kRound + 15.f)) & 15u) << (4 * (e & 1 ? 4 + e / 2 : e / 2));
    }
    if (!plain || worst > 0.4999f) {
        word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) word |= code_of(v[e], d, m) << (4 * (e & 1 ? 4 + e / 2 : e / 2));
    }
    return word;
}

}  // namespace svq
