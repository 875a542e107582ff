// Shared by the entry points for packed batches of tokens: element types and the caller's current
// device.
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/prep.h"

namespace prep {

// fp32 values in and out of an element type; every rounding is to nearest even
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__hip_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __hip_bfloat16 from_float<__hip_bfloat16>(float v) { return __float2bfloat16(v); }

inline int element_bytes(int dtype) { return dtype == PREP_F32 ? 4 : 2; }
inline bool float_type(int dtype) { return dtype == PREP_F32 || dtype == PREP_F16 || dtype == PREP_BF16; }
inline bool aligned(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// Launches `blocks` workgroups of `threads`: launch(first, n) for n of them from `first` on, in as many launches as it takes, since HIP takes
// fewer than 2^32 work-items along an axis.
template <typename Launch>
void in_launches(uint32_t blocks, int threads, const Launch &launch)
{
    const uint32_t most = 0xFFFFFFFFu / (uint32_t)threads;
    for (uint32_t first = 0, n; first < blocks; first += n) {
        n = blocks - first < most ? blocks - first : most;
        launch(first, n);
    }
}

// Makes `device` current and the caller's device current again at the end.
class DeviceScope {
public:
    explicit DeviceScope(int device)
    {
        int now = -1;
        if (hipGetDevice(&now) != hipSuccess) return;
        if (now == device) {
            ok_ = true;
            return;
        }
        if (hipSetDevice(device) != hipSuccess) return;
        ok_ = true;
        back_ = now;
    }
    ~DeviceScope()
    {
        if (back_ >= 0) (void)hipSetDevice(back_);
    }
    DeviceScope(const DeviceScope &) = delete;
    DeviceScope &operator=(const DeviceScope &) = delete;
    // on failure the runtime's error is taken back
    bool ok() const
    {
        if (!ok_) (void)hipGetLastError();
        return ok_;
    }

private:
    bool ok_ = false;
    int back_ = -1;
};

}  // namespace prep
