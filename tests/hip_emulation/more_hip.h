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
inline int __clz(int v) { return v == 0 ? 32 : __builtin_clz((unsigned)v); }

inline hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }

#define __builtin_amdgcn_fence(...) ((void)0)
// all lanes of the wave come here
inline void __builtin_amdgcn_wave_barrier()
{
    hip_emul::ThreadState &t = hip_emul::tls;
    t.ctx->wave_bar[t.tid.x >> 6]->arrive_and_wait();
}
