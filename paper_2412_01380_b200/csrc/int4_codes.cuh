// 4-bit codes (value = code - 8) as bfloat16 pairs, exactly, shared by the products that read them row by row.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

// Two values code - 8 from codes in the low four bits of either half of `codes`, whose other bits may be anything: in the low
// mantissa bits of 128 they are 128 + code.
__device__ __forceinline__ uint32_t int4_values(uint32_t codes)
{
    uint32_t v;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(v) : "r"(codes));
    const __nv_bfloat162 minus = __halves2bfloat162(__ushort_as_bfloat16(0xc308), __ushort_as_bfloat16(0xc308));       // -136
    __nv_bfloat162 b;
    b.x = __ushort_as_bfloat16((unsigned short)(v & 0xffffu));
    b.y = __ushort_as_bfloat16((unsigned short)(v >> 16));
    b = __hadd2(b, minus);
    return (uint32_t)__bfloat16_as_ushort(b.x) | ((uint32_t)__bfloat16_as_ushort(b.y) << 16);
}

// A word's eight codes as four pairs: codes 0 and 4, 1 and 5, 2 and 6, 3 and 7.
__device__ __forceinline__ void int4_pairs(uint32_t w, uint32_t (&v)[4])
{
#pragma unroll
    for (int s = 0; s < 4; ++s) v[s] = int4_values(w >> (4 * s));
}

// Four values, each rounded once to bfloat16.
__device__ __forceinline__ uint2 bf16x4(float a, float b, float c, float d)
{
    const __nv_bfloat162 lo = __floats2bfloat162_rn(a, b), hi = __floats2bfloat162_rn(c, d);
    return make_uint2((uint32_t)__bfloat16_as_ushort(lo.x) | ((uint32_t)__bfloat16_as_ushort(lo.y) << 16),
                      (uint32_t)__bfloat16_as_ushort(hi.x) | ((uint32_t)__bfloat16_as_ushort(hi.y) << 16));
}
