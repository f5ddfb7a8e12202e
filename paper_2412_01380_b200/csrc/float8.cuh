// Rounding of rows to their storage types, shared by what stages rows and what leaves them.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

// The scale of a block of 128 values with the largest magnitude amax: e4m3's largest value is 448.  Not below the smallest
// normal number, so that a block of zeros (or of values that vanish anyway) needs no case of its own.
__device__ __forceinline__ float fp8_scale(float amax) { return fmaxf(__fdiv_rn(amax, 448.f), 1.17549435e-38f); }

// rne(v / scale) as four e4m3 codes.  The quotient is rounded to binary32 first, as a definition by its formula has it: with a
// product by 1 / scale one code in some hundred of bfloat16 inputs, whose quotients often are exact ties, came out one step off.
__device__ __forceinline__ uint32_t fp8_codes4(float a, float b, float c, float d, float scale)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(__fdiv_rn(b, scale)), "f"(__fdiv_rn(a, scale)));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(__fdiv_rn(d, scale)), "f"(__fdiv_rn(c, scale)));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}

// Eight values, each rounded once to bfloat16.
__device__ __forceinline__ uint4 bf16x8(const float *v)
{
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        r[i] = (uint32_t)__bfloat16_as_ushort(b.x) | ((uint32_t)__bfloat16_as_ushort(b.y) << 16);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}
