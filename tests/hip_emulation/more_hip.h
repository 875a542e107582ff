// What the operators for packed batches of tokens use besides hip_runtime.h's stand-ins (test infrastructure).
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

struct float2 { float x, y; };

inline float __half2float(__half h)
{
    const uint32_t sign = (uint32_t)(h.x & 0x8000u) << 16, exp = (h.x >> 10) & 31u, man = h.x & 0x3FFu;
    uint32_t b = sign | (exp == 31 ? 0x7F800000u : (exp + 112u) << 23) | (man << 13);
    float f;
    if (exp == 0) {
        f = (float)man * (1.0f / 16777216.0f);
        memcpy(&b, &f, 4);
        b |= sign;
    }
    memcpy(&f, &b, 4);
    return f;
}

inline uint32_t atomicMax(uint32_t *p, uint32_t v)
{
    uint32_t old = __atomic_load_n(p, __ATOMIC_SEQ_CST);
    while (old < v && !__atomic_compare_exchange_n(p, &old, v, false, __ATOMIC_SEQ_CST, __ATOMIC_SEQ_CST)) {}
    return old;
}
inline uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }
inline int __clz(int v) { return v == 0 ? 32 : __builtin_clz((unsigned)v); }

inline hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }

#define __builtin_nontemporal_load(p) (*(p))
#define __builtin_nontemporal_store(v, p) (*(p) = (v))
#define __builtin_amdgcn_fence(...) ((void)0)
// all lanes of the wave come here
inline void __builtin_amdgcn_wave_barrier()
{
    hip_emul::ThreadState &t = hip_emul::tls;
    t.ctx->wave_bar[t.tid.x >> 6]->arrive_and_wait();
}

// csrc/matrix.h on the CPU: the same operands, products and sums in the order of the 32
#define PREP_MATRIX_H
namespace prep {
inline uint32_t byte_pair(uint32_t r0, uint32_t r1, int i) { return (r0 >> (8 * i) & 255u) | (r1 >> (8 * i) & 255u) << 16; }
constexpr float kBytePairScale = 1.0f / 16777216.0f;

inline float4 multiply_add_16x16x32(uint4 a, uint4 b, float4 c)
{
    hip_emul::ThreadState &t = hip_emul::tls;
    const unsigned lane = t.tid.x & 63;
    static uint32_t (*held)[64][8] = new uint32_t[16][64][8];  // of each wave: a and b of its lanes
    uint32_t (*mine)[8] = held[t.tid.x >> 6];
    const uint32_t own[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    memcpy(mine[lane], own, sizeof own);
    __builtin_amdgcn_wave_barrier();
    float r[4] = {c.x, c.y, c.z, c.w};
    for (unsigned i = 0; i < 4; i++)
        for (unsigned group = 0; group < 4; group++)
            for (unsigned k = 0; k < 8; k++) {
                const uint32_t *row = mine[16 * group + 4 * (lane / 16) + i], *col = mine[16 * group + lane % 16] + 4;
                const float x = __half2float(__half{(uint16_t)(row[k / 2] >> (16 * (k & 1)))});
                const float y = __half2float(__half{(uint16_t)(col[k / 2] >> (16 * (k & 1)))});
                r[i] += x * y;
            }
    __builtin_amdgcn_wave_barrier();
    return make_float4(r[0], r[1], r[2], r[3]);
}
}  // namespace prep
