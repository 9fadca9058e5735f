// Norm per head and rotation by position of queries and keys, in one pass over both; and its gradient.
//
//   n = x r,  r = 1 / sqrt(mean(x^2) + eps);     y = R (n w)        R turns the pairs of channels by the angles of the grid point
//   g = R^T dy;  dw = sum g n;  dx = r (g w - n mean(g w n))
//
// Bound by memory: x and y once (forward), x, dy and dx once (backward); nothing is kept between the passes, since r costs one
// reduction over channels that the backward pass holds in registers anyway.
//
// A vector of C channels is held by C / V neighbouring lanes (V channels of 16 bytes each; rounded up to a power of two), which sum by
// shuffles.  A group of lanes stays at a grid point and goes through the slices (batch and head): the point's cos and sin, 4 to 8 times
// the bytes of its channels, are read once for all of them.  Pairs lie within a lane if interleaved; else the partner is a shuffle
// away, or, if the pairs' distance is no multiple of V, in shared memory.
// In the backward pass a thread sums dw of its channels over all its vectors, a block over its threads, and a second kernel over the
// blocks in their order: no atomics.
#include <algorithm>

#include "sna_layer.cuh"

namespace sna {
namespace {

constexpr int ROTATE_THREADS = 256;
constexpr int MAX_PARTIALS = 148 * 8;       // blocks of one part in the backward pass, at most

enum class Pairs { IN_LANE, BY_SHUFFLE, BY_SHARED };

struct Strided { void* data; int64_t batch, head, lat, lon; };
struct Part {
    Strided x, y, dy;                   // backward: y is dx
    const float *weight, *lat_table, *lon_table;
    float* partials;                    // backward, if dweight is wanted: [blocks][C]
    int nlon, points, H, slices;        // slices = B * H
    int pairs_lat, pairs;
    int point_blocks, slice_blocks;     // the part's blocks: slice_blocks of point_blocks each
    int slices_per_block;
};
struct RotateArgs {
    Part part[2];
    int first_blocks;       // blocks of part 0; the others are part 1's
    int C, lanes;           // lanes of a vector: a power of two
    float eps;
};

__device__ __forceinline__ int64_t at(const Strided& t, int i, int j) { return i * t.lat + j * t.lon; }

template <typename T, int V, Pairs PAIRS, bool BACKWARD>
__global__ void __launch_bounds__(ROTATE_THREADS) norm_rotate_kernel(const __grid_constant__ RotateArgs a) {
    constexpr int U = 2;                // vectors of a group under way
    // (the last sum over threads needs room for a block's partial dw; the exchange for a block's vectors, one of U at a time)
    __shared__ __align__(16) float shared[ROTATE_THREADS * V];
    const int which = (int)blockIdx.x >= a.first_blocks;
    const Part& p = a.part[which];
    const int block = (int)blockIdx.x - (which ? a.first_blocks : 0);
    const int lane = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes, groups = ROTATE_THREADS / a.lanes;
    const int c0 = lane * V, C = a.C;
    const bool mine = c0 < C;
    const int P = p.pairs;
    float* row = shared + group * a.lanes * V;

    float w[V], dw[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        w[i] = mine && p.weight != nullptr ? p.weight[c0 + i] : 1.f;
        dw[i] = 0.f;
    }
    const int s_begin = (block / p.point_blocks) * p.slices_per_block, s_end = min(s_begin + p.slices_per_block, p.slices);
    const float inverse_C = 1.f / C;

    // the trips are the same for all groups of a block, whose lanes meet in shuffles; those beyond the last point do nothing
    for (int point0 = (block % p.point_blocks) * groups; point0 < p.points; point0 += p.point_blocks * groups) {
        const int point = point0 + group;
        const bool here = mine && point < p.points;
        const int i_lat = here ? point / p.nlon : 0, j_lon = here ? point - i_lat * p.nlon : 0;
        // y = cs * n + sn * partner; sn carries the sign of the pair's first channel
        float cs[V], sn[V];
        bool turned[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = c0 + i;
            const int pair = PAIRS == Pairs::IN_LANE ? c >> 1 : c < P ? c : c - P;
            const bool first = PAIRS == Pairs::IN_LANE ? (c & 1) == 0 : c < P;
            turned[i] = mine && c < 2 * P;
            cs[i] = 1.f; sn[i] = 0.f;
            if (turned[i]) {
                const float2 t = pair < p.pairs_lat ? reinterpret_cast<const float2*>(p.lat_table)[(int64_t)i_lat * p.pairs_lat + pair]
                                                    : reinterpret_cast<const float2*>(p.lon_table)[(int64_t)j_lon * (P - p.pairs_lat) + pair - p.pairs_lat];
                cs[i] = t.x;
                sn[i] = first ? -t.y : t.y;
            }
        }
        const T* x = static_cast<const T*>(p.x.data) + at(p.x, i_lat, j_lon) + c0;
        const T* dy = BACKWARD ? static_cast<const T*>(p.dy.data) + at(p.dy, i_lat, j_lon) + c0 : nullptr;
        T* y = static_cast<T*>(p.y.data) + at(p.y, i_lat, j_lon) + c0;
        int b = s_begin / p.H, h = s_begin - b * p.H;
        for (int s = s_begin; s < s_end; s += U) {
            Pack<T, V> xs[U], gs[U];
            int bs[U], hs[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                bs[u] = b; hs[u] = h;
                if (++h == p.H) { h = 0; ++b; }
                if (here && s + u < s_end) {
                    xs[u] = *reinterpret_cast<const Pack<T, V>*>(x + bs[u] * p.x.batch + hs[u] * p.x.head);
                    if (BACKWARD) gs[u] = *reinterpret_cast<const Pack<T, V>*>(dy + bs[u] * p.dy.batch + hs[u] * p.dy.head);
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) { xs[u].v[i] = from_float<T>(0.f); gs[u].v[i] = from_float<T>(0.f); }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // v: what the rotation acts on, n w (forward; without r, which is the same for the whole vector) or dy (backward)
                float xf[V], v[V], partner[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    xf[i] = to_float(xs[u].v[i]);
                    v[i] = BACKWARD ? to_float(gs[u].v[i]) : xf[i] * w[i];
                }
                if (PAIRS == Pairs::IN_LANE) {
#pragma unroll
                    for (int i = 0; i < V; ++i) partner[i] = v[i ^ 1];
                } else if (PAIRS == Pairs::BY_SHUFFLE) {
                    const int other = c0 < P ? lane + P / V : c0 < 2 * P ? lane - P / V : lane;
#pragma unroll
                    for (int i = 0; i < V; ++i) partner[i] = __shfl_sync(0xffffffffu, v[i], other, a.lanes);
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) row[c0 + i] = v[i];
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < V; ++i) { const int c = c0 + i; partner[i] = turned[i] ? row[c < P ? c + P : c - P] : 0.f; }
                    __syncwarp();
                }
                float square = 0.f, product = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    square = fmaf(xf[i], xf[i], square);
                    // (the transposed rotation has the other sign)
                    if (turned[i]) v[i] = BACKWARD ? fmaf(-sn[i], partner[i], cs[i] * v[i]) : fmaf(sn[i], partner[i], cs[i] * v[i]);
                    if (BACKWARD) product = fmaf(v[i] * w[i], xf[i], product);
                }
                for (int o = a.lanes / 2; o > 0; o >>= 1) {
                    square += __shfl_xor_sync(0xffffffffu, square, o);
                    if (BACKWARD) product += __shfl_xor_sync(0xffffffffu, product, o);
                }
                const float r = rsqrtf(square * inverse_C + a.eps);
                Pack<T, V> out;
                if (BACKWARD) {
                    // dx = r (g w - x r^2 sum(g w x) / C)
                    const float along = product * inverse_C * r * r;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        dw[i] = fmaf(v[i], xf[i] * r, dw[i]);
                        out.v[i] = from_float<T>(r * (v[i] * w[i] - xf[i] * along));
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) out.v[i] = from_float<T>(v[i] * r);
                }
                if (here && s + u < s_end) *reinterpret_cast<Pack<T, V>*>(y + bs[u] * p.y.batch + hs[u] * p.y.head) = out;
            }
        }
    }
    if (BACKWARD && p.partials != nullptr) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) shared[(group * a.lanes + lane) * V + i] = dw[i];      // lanes * V floats per group
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += ROTATE_THREADS) {
            float sum = 0.f;
            for (int g = 0; g < groups; ++g) sum += shared[g * a.lanes * V + c];
            p.partials[(int64_t)block * C + c] = sum;
        }
    }
}

struct SumArgs {
    const float* partials[2];
    float* dweight[2];
    int rows[2];
    int C;
};
// dweight = sum of the blocks' partial sums, in a fixed order.  One block per 32 channels and part; 32 rows of threads.
__global__ void __launch_bounds__(1024) sum_partials_kernel(const __grid_constant__ SumArgs a) {
    __shared__ float sums[32][33];
    const int which = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x;
    if (a.dweight[which] == nullptr) return;
    float sum = 0.f;
    if (c < a.C)
        for (int r = threadIdx.y; r < a.rows[which]; r += 32) sum += a.partials[which][(int64_t)r * a.C + c];
    sums[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.y == 0 && c < a.C) {
        float total = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) total += sums[r][threadIdx.x];
        a.dweight[which][c] = total;
    }
}

template <typename T, int V, bool BACKWARD>
cudaError_t launch_pairs(const RotateArgs& a, Pairs pairs, int blocks, cudaStream_t stream) {
    if (pairs == Pairs::IN_LANE) norm_rotate_kernel<T, V, Pairs::IN_LANE, BACKWARD><<<blocks, ROTATE_THREADS, 0, stream>>>(a);
    else if (pairs == Pairs::BY_SHUFFLE) norm_rotate_kernel<T, V, Pairs::BY_SHUFFLE, BACKWARD><<<blocks, ROTATE_THREADS, 0, stream>>>(a);
    else norm_rotate_kernel<T, V, Pairs::BY_SHARED, BACKWARD><<<blocks, ROTATE_THREADS, 0, stream>>>(a);
    return cudaGetLastError();
}
template <typename T>
cudaError_t launch_width(const RotateArgs& a, int V, Pairs pairs, bool backward, int blocks, cudaStream_t stream) {
    if constexpr (sizeof(T) == 2)
        if (V == 8) return backward ? launch_pairs<T, 8, true>(a, pairs, blocks, stream) : launch_pairs<T, 8, false>(a, pairs, blocks, stream);
    return backward ? launch_pairs<T, 4, true>(a, pairs, blocks, stream) : launch_pairs<T, 4, false>(a, pairs, blocks, stream);
}

// Largest power of two (up to 8) that divides the address in elements and all strides.
int granularity(const sna_tensor_t& t, size_t size) {
    const int64_t all = (int64_t)((uintptr_t)t.data / size) | t.batch | t.head | t.lat | t.lon | 8;
    return (uintptr_t)t.data % size != 0 ? 1 : (int)(all & -all);
}

sna_status_t norm_rotate(const sna_rotate_t* parts, int n_parts, sna_dtype_t dtype, int B, int C, float eps, int interleaved, bool backward,
                         void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    if (parts == nullptr || n_parts < 1 || n_parts > 2) return fail(SNA_ERR_INVALID_ARG, "one or two parts are needed");
    if (dtype != SNA_FLOAT32 && dtype != SNA_BFLOAT16 && dtype != SNA_FLOAT16) return fail(SNA_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
    if (B < 0) return fail(SNA_ERR_INVALID_ARG, "B must not be negative");
    if (C < 4 || C > 128 || C % 4 != 0) return fail(SNA_ERR_UNSUPPORTED, "C=%d unsupported (a multiple of 4 between 4 and 128)", C);
    if (!(eps >= 0.f)) return fail(SNA_ERR_INVALID_ARG, "eps must not be negative");
    int V = dtype != SNA_FLOAT32 && C % 8 == 0 ? 8 : 4;
    bool sums = false;
    for (int i = 0; i < n_parts; ++i) {
        const sna_rotate_t& r = parts[i];
        if (r.nlat < 0 || r.nlon < 0 || r.H < 0) return fail(SNA_ERR_INVALID_ARG, "sizes must not be negative");
        if ((int64_t)r.nlat * r.nlon > 0x3fffffff || (int64_t)B * r.H > 0x3fffffff) return fail(SNA_ERR_UNSUPPORTED, "nlat*nlon and B*H must be less than 2^30");
        if (r.pairs_lat < 0 || r.pairs_lon < 0 || r.pairs_lat > C || r.pairs_lon > C || 2 * (r.pairs_lat + r.pairs_lon) > C)
            return fail(SNA_ERR_INVALID_ARG, "%d + %d pairs do not fit into %d channels", r.pairs_lat, r.pairs_lon, C);
        sums = sums || (backward && r.dweight != nullptr);
        if ((int64_t)r.nlat * r.nlon * r.H * B == 0) continue;
        if ((r.pairs_lat > 0 && r.lat_table == nullptr) || (r.pairs_lon > 0 && r.lon_table == nullptr)) return fail(SNA_ERR_INVALID_ARG, "a table of angles is missing");
        if (((uintptr_t)r.lat_table | (uintptr_t)r.lon_table) & 7u) return fail(SNA_ERR_INVALID_ARG, "tables must be 8-byte aligned");
        if (((uintptr_t)r.weight | (uintptr_t)r.dweight) & 3u) return fail(SNA_ERR_INVALID_ARG, "weights must be 4-byte aligned");
        const sna_tensor_t* used[3] = {&r.x, backward ? &r.dx : &r.y, backward ? &r.dy : nullptr};
        for (const sna_tensor_t* t : used) {
            if (t == nullptr) continue;
            if (t->data == nullptr) return fail(SNA_ERR_INVALID_ARG, "a tensor's data is NULL");
            const int g = granularity(*t, size_of(dtype));
            if (g < 4) return fail(SNA_ERR_INVALID_ARG, "data pointers and strides must be multiples of 4 elements");
            if (g < V) V = 4;
        }
    }
    if (sums && (workspace == nullptr || ((uintptr_t)workspace & 15u))) return fail(SNA_ERR_INVALID_ARG, "workspace must be non-NULL and 16-byte aligned");
    if (sums && workspace_bytes < sna_norm_rotate_workspace_bytes(C))
        return fail(SNA_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", workspace_bytes, sna_norm_rotate_workspace_bytes(C));
    const int sms = sms_of_current_device();
    if (sms == 0) return fail(SNA_ERR_CUDA, "no CUDA device");

    RotateArgs a{};
    SumArgs sum{};
    a.C = C;
    a.eps = eps;
    a.lanes = 1;
    while (a.lanes * V < C) a.lanes *= 2;
    sum.C = C;
    int blocks[2] = {0, 0};
    Pairs pairs = interleaved ? Pairs::IN_LANE : Pairs::BY_SHUFFLE;
    for (int i = 0; i < n_parts; ++i) {
        const sna_rotate_t& r = parts[i];
        Part& p = a.part[i];
        auto strided = [](const sna_tensor_t& t) { return Strided{t.data, t.batch, t.head, t.lat, t.lon}; };
        p.x = strided(r.x);
        p.y = strided(backward ? r.dx : r.y);
        p.dy = strided(r.dy);
        p.weight = r.weight; p.lat_table = r.lat_table; p.lon_table = r.lon_table;
        p.nlon = std::max(r.nlon, 1); p.H = std::max(r.H, 1);
        p.points = r.nlat * r.nlon;
        p.slices = B * r.H;
        p.pairs_lat = r.pairs_lat; p.pairs = r.pairs_lat + r.pairs_lon;
        if (!interleaved && p.pairs % V != 0) pairs = Pairs::BY_SHARED;
        if (backward) sum.dweight[i] = r.dweight;
        if (p.points == 0 || p.slices == 0) continue;
        // A block's groups take neighbouring points.  Slices are spread over blocks until the GPU is full twice, as long as each still takes
        // four with the angles that it has read; the backward pass also bounds its blocks, each of which leaves a row of partial sums.
        const int groups = ROTATE_THREADS / a.lanes;
        p.point_blocks = (p.points + groups - 1) / groups;
        const int want = std::max(1, (2 * 8 * sms + p.point_blocks - 1) / p.point_blocks);
        p.slices_per_block = std::max(std::min(p.slices, 4), (p.slices + want - 1) / want);
        if (p.point_blocks < sms) p.slices_per_block = std::max(std::min(p.slices, 2), (p.slices + want - 1) / want);
        p.slice_blocks = (p.slices + p.slices_per_block - 1) / p.slices_per_block;
        if (backward && (int64_t)p.point_blocks * p.slice_blocks > MAX_PARTIALS) {
            p.slice_blocks = std::min(p.slice_blocks, MAX_PARTIALS);
            p.slices_per_block = (p.slices + p.slice_blocks - 1) / p.slice_blocks;
            p.slice_blocks = (p.slices + p.slices_per_block - 1) / p.slices_per_block;
            p.point_blocks = std::min(p.point_blocks, MAX_PARTIALS / p.slice_blocks);
        }
        const int64_t n = (int64_t)p.point_blocks * p.slice_blocks;
        if (n > 0x3fffffff) return fail(SNA_ERR_UNSUPPORTED, "problem too large");
        blocks[i] = (int)n;
        if (backward && r.dweight != nullptr) {
            p.partials = static_cast<float*>(workspace) + (size_t)i * MAX_PARTIALS * C;
            sum.partials[i] = p.partials;
            sum.rows[i] = blocks[i];
        }
    }
    a.first_blocks = blocks[0];
    const int total = blocks[0] + blocks[1];
    cudaError_t e = cudaSuccess;
    if (total > 0)
        e = dtype == SNA_FLOAT32    ? launch_width<float>(a, V, pairs, backward, total, stream)
            : dtype == SNA_BFLOAT16 ? launch_width<__nv_bfloat16>(a, V, pairs, backward, total, stream)
                                    : launch_width<__half>(a, V, pairs, backward, total, stream);
    if (e == cudaSuccess && sums) {
        sum_partials_kernel<<<dim3((C + 31) / 32, n_parts), dim3(32, 32), 0, stream>>>(sum);
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) return fail(SNA_ERR_CUDA, "norm and rotation launch: %s", cudaGetErrorString(e));
    return SNA_OK;
}

}  // namespace
}  // namespace sna

extern "C" {

size_t sna_norm_rotate_workspace_bytes(int C) { return C < 1 || C > 128 ? 0 : (size_t)2 * sna::MAX_PARTIALS * C * sizeof(float); }

sna_status_t sna_norm_rotate_forward(const sna_rotate_t* parts, int n_parts, sna_dtype_t dtype, int B, int C, float eps, int interleaved,
                                     void* cuda_stream) {
    return sna::norm_rotate(parts, n_parts, dtype, B, C, eps, interleaved, false, nullptr, 0, (cudaStream_t)cuda_stream);
}

sna_status_t sna_norm_rotate_backward(const sna_rotate_t* parts, int n_parts, sna_dtype_t dtype, int B, int C, float eps, int interleaved,
                                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return sna::norm_rotate(parts, n_parts, dtype, B, C, eps, interleaved, true, workspace, workspace_bytes, (cudaStream_t)cuda_stream);
}

}  // extern "C"
