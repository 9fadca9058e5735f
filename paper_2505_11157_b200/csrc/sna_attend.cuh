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

__host__ __device__ inline int64_t rows_of(const Problem& p) { return (int64_t)p.B * p.Hq * p.Nq; }

// Workspace of the backward pass: statistics per query, and the largest norms per key head (bits of floats)
struct Stats {
    float* lse2;                    // [B][Hq][Nq]: log2 of the sum of weights, +infinity for rows without any
    float* D;                       // [B][Hq][Nq]
    uint32_t* norms;                // [B][Hk][2]: of dout's rows, of v's rows (float16 only)
    uint4* extra;                   // [B][Hq][blocks of 64 queries][2][64]: what the tcgen05 dk/dv kernel adds to S and T per query (see there)
    uint4* weights;                 // [B or 1; B if there is a selection][blocks of 64 points][64]: what the tcgen05 dq kernel adds to S per point, if there are weights
    uint2* gone;                    // likewise, [blocks of 64 points]: bits of the points left out
};
constexpr int STATS_BLOCK = 64;

// The points that take part, one behind the other, for the tcgen05 kernels (workspace): where at least one point in sixteen of a batch is left out, its other
// keys and values are copied together first, so that the kernels walk as many points as there are.
struct Selection {
    int* taken;                     // [B]: the number of points, or Nk where they are read in place; null: no selection
    int* index;                     // [B][Nk]: which points they are
    float* weights;                 // [B][Nk]: their logarithmic weights
    void *k, *v;                    // [B][Hk][Nk][C]; zeros to the end of a tile of 128
};
constexpr int SELECT_POINTS = 256;
// It costs 3 us if few are left out, and a pass over the keys and values if many are; so not for small problems, nor where few rows share them, nor for so many
// points that counting them, which every block does, takes long.  us, forward and (in brackets) backward, B = 2, 8192 queries and points, bf16, with the points read
// in place : with a selection: 4 heads of 32, none left out 184 : 188 (421 : 421), 3 % 197 : 198 (476 : 471), 7 % 206 : 179 (516 : 409), 40 % 212 : 128 (530 : 301);
// 8 heads of 128 426 : 430 (1405 : 1400), 7 % 559 : 475 (1736 : 1474), 40 % 572 : 349 (1740 : 1086).  B = 1, 4 heads of 32, 2048 queries and points, none 19.5 : 21.7
// (82 : 85), 40 % 20.5 : 21.0 (80 : 83).
inline bool selects(const Problem& p) {
    return p.log_weights != nullptr && (int64_t)p.G * p.Nq >= 2048 && p.Nk <= 65536 && rows_of(p) * p.Nk >= (int64_t)1 << 27;
}
inline View selected_view(const Problem& p, void* data) { return View{data, (int64_t)p.Hk * p.Nk * p.C, (int64_t)p.Nk * p.C, p.C}; }
inline int64_t select_blocks_of(const Problem& p) { return (int64_t)p.B * p.Hk * ((p.Nk + SELECT_POINTS - 1) / SELECT_POINTS); }

__host__ __device__ inline int64_t weight_blocks_of(const Problem& p, bool selected) {
    return p.log_weights == nullptr ? 0 : (int64_t)(p.log_weights_batch == 0 && !selected ? 1 : p.B) * ((p.Nk + STATS_BLOCK - 1) / STATS_BLOCK);
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

// tcgen05 kernels (sna_kernels_attend_tc.cu).  False: the driver refuses a map of one of the tensors (heads that share memory, say).
// partials: room for partial_floats of the kernel.
enum class Kernel { FORWARD, DQ, DKDV };
Split split_of(const Problem& p, Kernel kernel, int sms);
size_t partial_floats(const Problem& p, Kernel kernel, int sms);
bool forward_tc(const Problem& p, const Selection& sel, sna_dtype_t dtype, int sms, float* partials, cudaStream_t stream, cudaError_t& e);
bool backward_tc(const Problem& p, const Stats& s, const Selection& sel, sna_dtype_t dtype, int sms, float* dq_partials, float* dkdv_partials, cudaStream_t stream, cudaError_t& e);
cudaError_t join_backward(const Problem& p, const Selection& sel, sna_dtype_t dtype, int sms, const float* dq_partials, const float* dkdv_partials, cudaStream_t stream);
cudaError_t read_status(int* status);
cudaError_t launch_wait_probe(cudaStream_t stream);

// mma.sync kernels (sna_kernels_attend.cu)
int forward_splits(const Problem& p, int sms);
cudaError_t launch_join(const Problem& p, sna_dtype_t dtype, int splits, const float* partials, cudaStream_t stream);
cudaError_t launch_forward(const Problem& p, sna_dtype_t dtype, int splits, float* partials, cudaStream_t stream);
cudaError_t launch_statistics(const Problem& p, const Stats& s, const Selection& sel, sna_dtype_t dtype, cudaStream_t stream);      // and the selection
cudaError_t launch_selection(const Problem& p, const Selection& sel, cudaStream_t stream);
cudaError_t launch_backward_dq(const Problem& p, const Stats& s, sna_dtype_t dtype, cudaStream_t stream);
cudaError_t launch_backward_dkdv(const Problem& p, const Stats& s, sna_dtype_t dtype, cudaStream_t stream);

}  // namespace attend
}  // namespace sna
