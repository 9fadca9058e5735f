// What the operators around the attention of a layer share: 16-bit types, errors, the state of a device.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <utility>

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
// Kernels of one call that follow each other: a dependent may be set up while the kernel before it ends.  It calls wait_for_previous before it reads what that
// kernel (and so every one before) has written, and at the latest at its end; the kernel before calls allow_dependents.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void allow_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <typename... Parameters, typename... Arguments>
cudaError_t launch_dependent(void (*kernel)(Parameters...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, Arguments&&... arguments) {
    cudaLaunchAttribute attribute{};
    attribute.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attribute.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = grid; config.blockDim = block; config.dynamicSmemBytes = smem; config.stream = stream;
    config.attrs = &attribute; config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, std::forward<Arguments>(arguments)...);
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// Packed fp32 pairs: one instruction for two lanes of a 64-bit register pair
__device__ __forceinline__ uint64_t pack2(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) { uint64_t d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }

// The V values of a lane as 32-bit words, and as packed pairs of fp32
template <typename T, int V> struct Words {
    static constexpr int N = (int)sizeof(T) * V / 4;
    uint32_t w[N];
};
template <typename T> __device__ __forceinline__ uint64_t pair_of(uint32_t word);
template <> __device__ __forceinline__ uint64_t pair_of<__nv_bfloat16>(uint32_t word) { return pack2(__uint_as_float(word << 16), __uint_as_float(word & 0xffff0000u)); }
template <> __device__ __forceinline__ uint64_t pair_of<__half>(uint32_t word) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&word));
    return pack2(f.x, f.y);
}
template <typename T> __device__ __forceinline__ uint32_t word_of(float lo, float hi);
template <> __device__ __forceinline__ uint32_t word_of<__nv_bfloat16>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t word_of<__half>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <typename T, int V> __device__ __forceinline__ void pairs_of(const Words<T, V>& x, uint64_t (&f)[V / 2]) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        if constexpr (sizeof(T) == 4) f[i] = pack2(__uint_as_float(x.w[2 * i]), __uint_as_float(x.w[2 * i + 1]));
        else f[i] = pair_of<T>(x.w[i]);
    }
}
template <typename T, int V> __device__ __forceinline__ Words<T, V> words_of(const uint64_t (&f)[V / 2]) {
    Words<T, V> x;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        float a, b;
        unpack2(f[i], a, b);
        if constexpr (sizeof(T) == 4) { x.w[2 * i] = __float_as_uint(a); x.w[2 * i + 1] = __float_as_uint(b); }
        else {
            x.w[i] = word_of<T>(a, b);
        }
    }
    return x;
}
template <typename T, int V> __device__ __forceinline__ Words<T, V> load_words(const T* p) {
    Words<T, V> x;
    if constexpr (Words<T, V>::N == 4) { const uint4 q = *reinterpret_cast<const uint4*>(p); x.w[0] = q.x; x.w[1] = q.y; x.w[2] = q.z; x.w[3] = q.w; }
    else { const uint2 q = *reinterpret_cast<const uint2*>(p); x.w[0] = q.x; x.w[1] = q.y; }
    return x;
}
template <typename T, int V> __device__ __forceinline__ void store_words(T* p, const Words<T, V>& x) {
    if constexpr (Words<T, V>::N == 4) *reinterpret_cast<uint4*>(p) = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(x.w[0], x.w[1]);
}
// V values in one load or store
template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };
#endif

}  // namespace sna
