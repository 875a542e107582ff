// The matrix instruction that the patch rows use, and its operands (gfx950).
#ifndef PREP_MATRIX_H
#define PREP_MATRIX_H
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace prep {

// The values of byte i of r0 and of r1, times 2^-24, as two halves: a half whose low byte is b and whose high byte is 0 is the
// subnormal b 2^-24, which the product below takes as it is.
__device__ __forceinline__ uint32_t byte_pair(uint32_t r0, uint32_t r1, int i)
{
    return __builtin_amdgcn_perm(r1, r0, 0x0C040C00u + (uint32_t)i * 0x00010001u);
}
constexpr float kBytePairScale = 1.0f / 16777216.0f;

// c + a b, fp32 sums of products of halves.  a: 16 rows of 32, lane l holds eight values of row l mod 16; b: 32 of 16 columns, lane l
// holds eight values of column l mod 16; which eight of the 32 a lane holds depends on l / 16 alone, in the same way for both.  c and
// the result: lane l holds column l mod 16 of rows 4 (l / 16) .. + 3.
__device__ __forceinline__ float4 multiply_add_16x16x32(uint4 a, uint4 b, float4 c)
{
    typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
    typedef float Float4 __attribute__((ext_vector_type(4)));
    const Float4 sum = {c.x, c.y, c.z, c.w};
    const Float4 r = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Half8, a), __builtin_bit_cast(Half8, b), sum, 0, 0, 0);
    return make_float4(r.x, r.y, r.z, r.w);
}

}  // namespace prep
#endif
