// Dropout into a residual, with random numbers from a counter: Philox 4x32 with ten rounds, from the definition in Salmon et al.,
// "Parallel random numbers: as easy as 1, 2, 3" (SC 2011).
//
// A round multiplies two of the counter's four words by constants and mixes the high halves with the others and the key; the block for
// counter (e / 4, offset) decides about the elements e .. e + 3, so any thread can draw for any element and the backward pass draws the
// same numbers again: no mask is stored, which would cost an eighth of a byte or more per element both ways.
//
// Bound by memory: x, residual, out once each (16-bit: 6 bytes per element), about 18 instructions per element of the 33 that the issue slots
// allow at that rate.  A thread takes two packs of 16 bytes, all their loads issued before the first round.
#include "sna_layer.cuh"

namespace sna {
namespace {

constexpr int DROPOUT_THREADS = 256;
constexpr int PACKS = 2;        // per thread and array

__device__ __forceinline__ void philox(uint64_t block, uint64_t offset, uint64_t seed, uint32_t (&word)[4]) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    word[0] = c0; word[1] = c1; word[2] = c2; word[3] = c3;
}

// Elements [first, first + V) of one pack; V is a multiple of 4, or 1.
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> drop(const Pack<T, V>& x, const Pack<T, V>& residual, bool has_residual, int64_t first,
                                           uint64_t seed, uint64_t offset, uint32_t threshold, float scale) {
    Pack<T, V> out;
    uint32_t word[4];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (i % 4 == 0) philox((uint64_t)(first + i) >> 2, offset, seed, word);
        const uint32_t drawn = V > 1 ? word[i % 4] : (first & 2) ? ((first & 1) ? word[3] : word[2]) : ((first & 1) ? word[1] : word[0]);
        // (chosen, not multiplied by zero: what is dropped may be infinite or NaN)
        float y = drawn >= threshold ? to_float(x.v[i]) * scale : 0.f;
        if (has_residual) y += to_float(residual.v[i]);
        out.v[i] = from_float<T>(y);
    }
    return out;
}

template <typename T, int V>
__global__ void __launch_bounds__(DROPOUT_THREADS) dropout_kernel(const T* x, const T* residual, T* out, int64_t n, uint32_t threshold,
                                                                  float scale, const int64_t* __restrict__ rng) {
    const uint64_t seed = (uint64_t)rng[0], offset = (uint64_t)rng[1];
    const int64_t block_first = (int64_t)blockIdx.x * (DROPOUT_THREADS * V * PACKS);
    Pack<T, V> a[PACKS], r[PACKS];
    if (block_first + DROPOUT_THREADS * V * PACKS <= n) {
#pragma unroll
        for (int j = 0; j < PACKS; ++j) {
            const int64_t first = block_first + (j * DROPOUT_THREADS + threadIdx.x) * V;
            a[j] = *reinterpret_cast<const Pack<T, V>*>(x + first);
            if (residual != nullptr) r[j] = *reinterpret_cast<const Pack<T, V>*>(residual + first);
        }
#pragma unroll
        for (int j = 0; j < PACKS; ++j) {
            const int64_t first = block_first + (j * DROPOUT_THREADS + threadIdx.x) * V;
            *reinterpret_cast<Pack<T, V>*>(out + first) = drop<T, V>(a[j], r[j], residual != nullptr, first, seed, offset, threshold, scale);
        }
        return;
    }
    for (int64_t e = block_first + threadIdx.x; e < n && e < block_first + DROPOUT_THREADS * V * PACKS; e += DROPOUT_THREADS) {
        Pack<T, 1> xe, re;
        xe.v[0] = x[e];
        if (residual != nullptr) re.v[0] = residual[e];
        out[e] = drop<T, 1>(xe, re, residual != nullptr, e, seed, offset, threshold, scale).v[0];
    }
}

template <typename T, int V>
cudaError_t launch(const void* x, const void* residual, void* out, int64_t n, uint32_t threshold, float scale, const int64_t* rng, cudaStream_t stream) {
    const int64_t per_block = (int64_t)DROPOUT_THREADS * V * PACKS, blocks = (n + per_block - 1) / per_block;
    dropout_kernel<T, V><<<(unsigned)blocks, DROPOUT_THREADS, 0, stream>>>((const T*)x, (const T*)residual, (T*)out, n, threshold, scale, rng);
    return cudaGetLastError();
}

// Packs of 16 bytes where every pointer allows it; single elements otherwise (a view that starts in the middle of a tensor).
template <typename T>
cudaError_t launch_dropout(const void* x, const void* residual, void* out, int64_t n, uint32_t threshold, float scale, const int64_t* rng, cudaStream_t stream) {
    const bool aligned = (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)out) & 15u) == 0;
    return aligned ? launch<T, 16 / sizeof(T)>(x, residual, out, n, threshold, scale, rng, stream)
                   : launch<T, 1>(x, residual, out, n, threshold, scale, rng, stream);
}

}  // namespace
}  // namespace sna

extern "C" sna_status_t sna_dropout(const void* x, const void* residual, void* out, sna_dtype_t dtype, int64_t n, double p,
                                    const int64_t* rng, void* cuda_stream) {
    using sna::fail;
    if (dtype != SNA_FLOAT32 && dtype != SNA_BFLOAT16 && dtype != SNA_FLOAT16) return fail(SNA_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
    if (!(p >= 0.0 && p < 1.0)) return fail(SNA_ERR_INVALID_ARG, "p must be at least 0 and less than 1");
    if (n < 0) return fail(SNA_ERR_INVALID_ARG, "n must not be negative");
    if (n >= ((int64_t)1 << 39)) return fail(SNA_ERR_UNSUPPORTED, "n must be less than 2^39");      // the grid of single elements
    if (n == 0) return SNA_OK;
    if (!x || !out || !rng) return fail(SNA_ERR_INVALID_ARG, "x, out and rng must not be NULL");
    if ((((uintptr_t)x | (uintptr_t)residual | (uintptr_t)out) & (sna::size_of(dtype) - 1)) || ((uintptr_t)rng & 7u))
        return fail(SNA_ERR_INVALID_ARG, "device pointers must be aligned to their elements");
    const double threshold = nearbyint(p * 4294967296.0);
    const uint32_t least = threshold > 4294967295.0 ? 4294967295u : (uint32_t)threshold;
    const float scale = (float)(1.0 / (1.0 - p));
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const cudaError_t e = dtype == SNA_FLOAT32    ? sna::launch_dropout<float>(x, residual, out, n, least, scale, rng, stream)
                          : dtype == SNA_BFLOAT16 ? sna::launch_dropout<__nv_bfloat16>(x, residual, out, n, least, scale, rng, stream)
                                                  : sna::launch_dropout<__half>(x, residual, out, n, least, scale, rng, stream);
    if (e != cudaSuccess) return fail(SNA_ERR_CUDA, "dropout launch: %s", cudaGetErrorString(e));
    return SNA_OK;
}
