// 4-bit codes (value = code - 8) as bfloat16 pairs, exactly, shared by the products that read them row by row.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

// A word's eight codes as four pairs, codes 0 and 4, 1 and 5, 2 and 6, 3 and 7: all of them (code - 8) / 64.  A bfloat16 whose upper eight bits are
// zero is its lower eight, as a number, times 2^-133 (the smallest normal numbers go on where the subnormal ones end), so a code need not be moved
// within its byte: one AND brings a pair out, one multiply-add by 2^127, or, for the upper half of a byte, 2^123, makes it code / 64 - 8 / 64.  (Of a
// step's logic and shifts, which run at half the rate of multiply-adds and bound the product of few rows, this leaves 5 for 8 codes instead of 7.)
__device__ __forceinline__ void int4_pairs(uint32_t w, uint32_t (&v)[4])
{
    const uint32_t h = w >> 8;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[0]) : "r"(w & 0x000f000fu), "r"(0x7f007f00u), "r"(0xbe00be00u));    // * 2^127 - 1/8
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[1]) : "r"(w & 0x00f000f0u), "r"(0x7d007d00u), "r"(0xbe00be00u));    // * 2^123 - 1/8
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[2]) : "r"(h & 0x000f000fu), "r"(0x7f007f00u), "r"(0xbe00be00u));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[3]) : "r"(h & 0x00f000f0u), "r"(0x7d007d00u), "r"(0xbe00be00u));
}
// The same word as four pairs of neighbours (codes 0 and 1, 2 and 3, ...), all of them (code - 8) / 64, for operands that are in order.
__device__ __forceinline__ void int4_in_order(uint32_t w, uint32_t *v)
{
    const uint32_t lo = w & 0x0f0f0f0fu, hi = w & 0xf0f0f0f0u;       // (a byte's codes stay where they are in it)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        // byte j of lo, nothing, byte j of hi, nothing: "nothing" is the upper bit of lo's byte, all over
        uint32_t both;
        asm("prmt.b32 %0, %1, %2, %3;" : "=r"(both) : "r"(lo), "r"(hi), "r"(0x8480 + 0x1111 * j));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[j]) : "r"(both), "r"(0x7d007f00u), "r"(0xbe00be00u));      // * (2^127, 2^123) - 1/8
    }
}
// A product by these operands times this is the product.  (It goes into the scale, where it is exact: sums of 1/64 of what they stand for lose the
// last bits of outputs near binary32's smallest normal number.  The products themselves are multiples of 2^-139, which binary32 holds.)
constexpr float INT4_PRODUCT = 64.f;

// Four values, each rounded once to bfloat16.
__device__ __forceinline__ uint2 bf16x4(float a, float b, float c, float d)
{
    const __nv_bfloat162 lo = __floats2bfloat162_rn(a, b), hi = __floats2bfloat162_rn(c, d);
    return make_uint2((uint32_t)__bfloat16_as_ushort(lo.x) | ((uint32_t)__bfloat16_as_ushort(lo.y) << 16),
                      (uint32_t)__bfloat16_as_ushort(hi.x) | ((uint32_t)__bfloat16_as_ushort(hi.y) << 16));
}
