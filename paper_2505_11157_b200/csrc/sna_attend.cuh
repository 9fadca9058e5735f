// What the 16-bit attention's kernels and their dispatch share.
#pragma once
#include "sna_layer.cuh"

namespace sna {
namespace attend {

// Logarithmic weights that are not above this leave their point out (the lowest numbers of 32 and of 16 bits count as -infinity do).
constexpr float EXCLUDED = -1e30f;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// [B][H][points][C]: strides in elements
struct View {
    void* data;
    int64_t batch, head, point;
};

struct Problem {
    View q, k, v, out, rest, dout, dq, dk, dv;      // rest: what rounding took from out; its data may be null
    float* lse;                     // [B][Hq][Nq], natural logarithm; may be null in the forward pass
    const float* log_weights;       // [B or 1][Nk], or null
    int64_t log_weights_batch;      // 0: shared
    int B, Hq, Hk, G, Nq, Nk, C;    // G = Hq / Hk
    float scale, scale_log2;
};

// Workspace of the backward pass: statistics per query, and the largest norms per key head (bits of floats)
struct Stats {
    float* lse2;                    // [B][Hq][Nq]: log2 of the sum of weights, +infinity for rows without any
    float* D;                       // [B][Hq][Nq]
    uint32_t* norms;                // [B][Hk][2]: of dout's rows, of v's rows (float16 only)
    uint4* extra;                   // [B][Hq][blocks of 64 queries][2][64]: what the tcgen05 dk/dv kernel adds to S and T per query (see there)
    uint4* weights;                 // [B or 1][blocks of 64 points][64]: what the tcgen05 dq kernel adds to S per point, if there are weights
    uint2* gone;                    // [B or 1][blocks of 64 points]: bits of the points left out
};
constexpr int STATS_BLOCK = 64;
__host__ __device__ inline int64_t weight_blocks_of(const Problem& p) {
    return p.log_weights == nullptr ? 0 : (int64_t)(p.log_weights_batch == 0 ? 1 : p.B) * ((p.Nk + STATS_BLOCK - 1) / STATS_BLOCK);
}

// How a tcgen05 kernel's tiles become thread blocks, of which an SM runs one at a time: the first `full` tiles whole, the others in `parts` pieces of the
// streamed side, whose partial results (fp32) a second kernel joins.
// The whole waves stay whole.  The last, partial wave is cut so that its pieces end early: R tiles in k pieces take ceil(R k / SMs) / k of a wave (256 tiles on 148
// SMs: 1.75 waves with four pieces each instead of 2).  Not for many waves, which gain little, nor into pieces of a few streamed blocks.
struct Split {
    int64_t tiles, full;
    int parts;
    __host__ __device__ int64_t blocks() const { return full + (tiles - full) * parts; }
    __host__ __device__ int64_t rest() const { return tiles - full; }
};
__host__ __device__ inline int64_t query_blocks_of(const Problem& p) { return (int64_t)p.B * p.Hq * ((p.Nq + STATS_BLOCK - 1) / STATS_BLOCK); }

// Powers of two that keep float16 operands of the second products away from the numbers that its exponent has no room for: softmax
// weights (at most 1) and, in the backward pass, probabilities are held times 2^SHIFT.
template <typename T> constexpr float SHIFT = 0.f;
template <> constexpr float SHIFT<__half> = 14.f;

#ifdef __CUDACC__
// A number in three bfloat16 parts (24 bits), whose products with ones a tensor core adds up.
constexpr uint32_t EXTRA_ONES_0 = 0x3f803f80u, EXTRA_ONES_1 = 0x00003f80u;
constexpr uint32_t EXTRA_OUT = 0x0000ff61u;        // -2.99e38: times a scale of 2^-20 or more, below any finite score of a point that takes part
__device__ __forceinline__ uint2 extra_parts(float x) {
    const __nv_bfloat16 hi = __float2bfloat16_rn(x);
    const float rest = x - __bfloat162float(hi);
    const __nv_bfloat16 mid = __float2bfloat16_rn(rest), lo = __float2bfloat16_rn(rest - __bfloat162float(mid));
    return make_uint2((uint32_t)__bfloat16_as_ushort(hi) | ((uint32_t)__bfloat16_as_ushort(mid) << 16), __bfloat16_as_ushort(lo));
}

// The power of two that ds is held times.  The probabilities in it are already held times 2^SHIFT; with |t - D| <= bound the products stay below 2^15.
template <typename T>
__device__ __forceinline__ float ds_scale(const Stats& s, int bk) {
    if (SHIFT<T> == 0.f) return 1.f;
    const float bound = 2.f * __uint_as_float(s.norms[bk * 2]) * __uint_as_float(s.norms[bk * 2 + 1]);
    if (!(bound > 0.f && bound < INFINITY)) return 1.f;
    return exp2f(fminf(fmaxf(-ceilf(log2f(bound)), -100.f), 100.f));
}
#endif

inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }
__host__ __device__ inline int64_t rows_of(const Problem& p) { return (int64_t)p.B * p.Hq * p.Nq; }

// tcgen05 kernels (sna_kernels_attend_tc.cu).  False: the driver refuses a map of one of the tensors (heads that share memory, say).
// partials: room for partial_floats of the kernel.
enum class Kernel { FORWARD, DQ, DKDV };
Split split_of(const Problem& p, Kernel kernel, int sms);
size_t partial_floats(const Problem& p, Kernel kernel, int sms);
bool forward_tc(const Problem& p, sna_dtype_t dtype, int sms, float* partials, cudaStream_t stream, cudaError_t& e);
bool backward_dq_tc(const Problem& p, const Stats& s, sna_dtype_t dtype, int sms, float* partials, cudaStream_t stream, cudaError_t& e);
bool backward_dkdv_tc(const Problem& p, const Stats& s, sna_dtype_t dtype, int sms, float* partials, cudaStream_t stream, cudaError_t& e);
cudaError_t join_backward(const Problem& p, sna_dtype_t dtype, int sms, const float* dq_partials, const float* dkdv_partials, cudaStream_t stream);
cudaError_t read_status(int* status);
cudaError_t launch_wait_probe(cudaStream_t stream);

// mma.sync kernels (sna_kernels_attend.cu)
int forward_splits(const Problem& p, int sms);
cudaError_t launch_join(const Problem& p, sna_dtype_t dtype, int splits, const float* partials, cudaStream_t stream);
cudaError_t launch_forward(const Problem& p, sna_dtype_t dtype, int splits, float* partials, cudaStream_t stream);
cudaError_t launch_statistics(const Problem& p, const Stats& s, sna_dtype_t dtype, cudaStream_t stream);
cudaError_t launch_backward_dq(const Problem& p, const Stats& s, sna_dtype_t dtype, cudaStream_t stream);
cudaError_t launch_backward_dkdv(const Problem& p, const Stats& s, sna_dtype_t dtype, cudaStream_t stream);

}  // namespace attend
}  // namespace sna
