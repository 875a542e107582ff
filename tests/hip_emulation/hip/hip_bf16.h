// CPU stand-in for the bfloat16 conversions libprep uses (test infrastructure).
#pragma once
#include <cstdint>
#include <cstring>

struct __hip_bfloat16 { uint16_t x; };

// round to nearest even; NaN stays NaN
inline __hip_bfloat16 __float2bfloat16(float f)
{
    uint32_t b;
    memcpy(&b, &f, 4);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return __hip_bfloat16{(uint16_t)((b >> 16) | 0x40u)};
    return __hip_bfloat16{(uint16_t)((b + 0x7FFFu + ((b >> 16) & 1u)) >> 16)};
}
inline float __bfloat162float(__hip_bfloat16 v)
{
    const uint32_t b = (uint32_t)v.x << 16;
    float f;
    memcpy(&f, &b, 4);
    return f;
}
