// Dropout into a residual, with random numbers from a counter: Philox 4x32 with ten rounds, from the definition in Salmon et al.,
// "Parallel random numbers: as easy as 1, 2, 3" (SC 2011).
//
// A round multiplies two of the counter's four words by constants and mixes the high halves with the others and the key; the block for
// counter (e / 4, offset) decides about the elements e .. e + 3, so any thread can draw for any element and the backward pass draws the
// same numbers again: no mask is stored, which would cost an eighth of a byte or more per element both ways.
//
// x, residual and out are moved once each (16-bit: 6 bytes per element), but the generator's 32-bit products bound it before the memory does: 36 of them per eight
// elements keep the integer-multiply pipe 68 to 73 % busy, 212 instructions per eight elements the issue slots 61 to 64 %.  4 x 128x256 x 256 bf16: 44 us
// forward (4.5 TB/s), 41 backward (3.3 TB/s).
// A thread takes one pack of 16 bytes, or two where there is work enough (the same size: one 95 us, two 86, four 86; 3 x 91x181 x 77: 16, 21, 20).
#include "sna_layer.cuh"

namespace sna {
namespace {

constexpr int DROPOUT_THREADS = 256;

__device__ __forceinline__ void philox(uint32_t block_low, uint32_t block_high, uint64_t offset, uint64_t seed, uint32_t (&word)[4]) {
    uint32_t c0 = block_low, c1 = block_high, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
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

// Elements [first, first + V) of one pack, V a multiple of 4.  `high`: the high word of first / 4, the same for a whole thread block (whose elements
// begin at a multiple of their number): what the first rounds compute from it and from the offset alone is then computed once per thread.
template <typename T, int V>
__device__ __forceinline__ Words<T, V> drop(const Words<T, V>& x, const Words<T, V>& residual, bool has_residual, int64_t first, uint32_t high,
                                            uint64_t seed, uint64_t offset, uint32_t threshold, float scale) {
    uint64_t f[V / 2], r[V / 2];
    pairs_of<T, V>(x, f);
    if (has_residual) pairs_of<T, V>(residual, r);
    uint32_t word[4];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        if (i % 2 == 0) philox((uint32_t)((uint64_t)first >> 2) + i / 2, high, offset, seed, word);
        float a, b;
        unpack2(f[i], a, b);
        // (chosen, not multiplied by zero: what is dropped may be infinite or NaN)
        f[i] = pack2(word[2 * (i % 2)] >= threshold ? a : 0.f, word[2 * (i % 2) + 1] >= threshold ? b : 0.f);
        f[i] = has_residual ? fma2(f[i], pack2(scale, scale), r[i]) : mul2(f[i], pack2(scale, scale));
    }
    return words_of<T, V>(f);
}
// a single element
template <typename T>
__device__ __forceinline__ T drop_one(T x, T residual, bool has_residual, int64_t e, uint64_t seed, uint64_t offset, uint32_t threshold, float scale) {
    uint32_t word[4];
    philox((uint32_t)((uint64_t)e >> 2), (uint32_t)((uint64_t)e >> 34), offset, seed, word);
    const uint32_t drawn = (e & 2) ? ((e & 1) ? word[3] : word[2]) : ((e & 1) ? word[1] : word[0]);
    const float kept = drawn >= threshold ? to_float(x) : 0.f;
    return from_float<T>(has_residual ? fmaf(kept, scale, to_float(residual)) : kept * scale);
}

template <typename T, int V, int PACKS>
__global__ void __launch_bounds__(DROPOUT_THREADS) dropout_kernel(const T* x, const T* residual, T* out, int64_t n, uint32_t threshold,
                                                                  float scale, const int64_t* __restrict__ rng) {
    const uint64_t seed = (uint64_t)rng[0], offset = (uint64_t)rng[1];
    const int64_t block_first = (int64_t)blockIdx.x * (DROPOUT_THREADS * V * PACKS);
    if constexpr (V > 1) {
        if (block_first + DROPOUT_THREADS * V * PACKS <= n) {
            const uint32_t high = (uint32_t)((uint64_t)block_first >> 34);
            Words<T, V> a[PACKS], r[PACKS];
#pragma unroll
            for (int j = 0; j < PACKS; ++j) {
                const int64_t first = block_first + (j * DROPOUT_THREADS + threadIdx.x) * V;
                a[j] = load_words<T, V>(x + first);
                if (residual != nullptr) r[j] = load_words<T, V>(residual + first);
            }
#pragma unroll
            for (int j = 0; j < PACKS; ++j) {
                const int64_t first = block_first + (j * DROPOUT_THREADS + threadIdx.x) * V;
                store_words<T, V>(out + first, drop<T, V>(a[j], r[j], residual != nullptr, first, high, seed, offset, threshold, scale));
            }
            return;
        }
    }
    for (int64_t e = block_first + threadIdx.x; e < n && e < block_first + DROPOUT_THREADS * V * PACKS; e += DROPOUT_THREADS)
        out[e] = drop_one<T>(x[e], residual != nullptr ? residual[e] : x[e], residual != nullptr, e, seed, offset, threshold, scale);
}

template <typename T, int V, int PACKS>
cudaError_t launch(const void* x, const void* residual, void* out, int64_t n, uint32_t threshold, float scale, const int64_t* rng, cudaStream_t stream) {
    const int64_t per_block = (int64_t)DROPOUT_THREADS * V * PACKS, blocks = (n + per_block - 1) / per_block;
    dropout_kernel<T, V, PACKS><<<(unsigned)blocks, DROPOUT_THREADS, 0, stream>>>((const T*)x, (const T*)residual, (T*)out, n, threshold, scale, rng);
    return cudaGetLastError();
}

// Packs of 16 bytes where every pointer allows it; single elements otherwise (a view that starts in the middle of a tensor).
template <typename T>
cudaError_t launch_dropout(const void* x, const void* residual, void* out, int64_t n, uint32_t threshold, float scale, const int64_t* rng, cudaStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    const bool aligned = (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)out) & 15u) == 0;
    if (!aligned) return launch<T, 1, 2>(x, residual, out, n, threshold, scale, rng, stream);
    return n < (int64_t)1 << 23 ? launch<T, V, 1>(x, residual, out, n, threshold, scale, rng, stream) : launch<T, V, 2>(x, residual, out, n, threshold, scale, rng, stream);
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
