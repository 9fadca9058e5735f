// What the operators around the attention of a layer share: 16-bit types, errors, the state of a device.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "../../include/sna.h"

namespace sna {

// Records the message of a failing call and returns its status (sna_api.cu).
sna_status_t fail(sna_status_t status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// Number of SMs of the current device; 0 if there is none.  (Looked up once per device: cudaDeviceGetAttribute is cheap, cudaGetDevice cheaper.)
inline int sms_of_current_device() {
    static std::atomic<int> known[64];
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0) return 0;
    if (device < 64)
        if (const int sms = known[device].load(std::memory_order_relaxed); sms != 0) return sms;
    int sms = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return 0;
    if (device < 64) known[device].store(sms, std::memory_order_relaxed);
    return sms;
}

inline size_t size_of(sna_dtype_t t) { return t == SNA_FLOAT32 ? 4 : 2; }

#ifdef __CUDACC__
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// V values in one load or store
template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };
#endif

}  // namespace sna
