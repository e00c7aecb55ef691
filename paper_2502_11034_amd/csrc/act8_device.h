// The checkpoint format's arithmetic: e4m3 codes of 32 values that share a power of two.
#ifndef ADAGC_ACT8_DEVICE_H
#define ADAGC_ACT8_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace adagc {

constexpr int kAct8LeastExponent = -100;   // what is below 2^-110 is 0; every value a checkpoint holds is a normal bf16 or fp32 number

// 2^e for e in -126 .. 127
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The smallest e with largest / 2^e <= 448 = 1.75 * 2^8, from the bits of a finite fp32 value: its exponent less 8, and one more
// where its significand is over 1.75.
__device__ __forceinline__ int act8_exponent(uint32_t largest)
{
    const int e = (int)((largest + 0x1FFFFFu) >> 23) - 127 - 8;
    return e < kAct8LeastExponent ? kAct8LeastExponent : e;
}

// Four codes of values already divided by the scale: finite ones are at most 448.
__device__ __forceinline__ uint32_t act8_encode(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}

}  // namespace adagc
#endif
