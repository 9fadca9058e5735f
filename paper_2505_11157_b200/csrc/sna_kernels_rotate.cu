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

// Walks the slices (batch, head) of a tensor by additions.
struct Walk {
    int64_t head, wrap;         // to the next head, and from the last head to the next batch's first
    int h, H;
    __device__ __forceinline__ Walk(const Strided& t, int h, int H) : head(t.head), wrap(t.batch - (H - 1) * t.head), h(h), H(H) {}
    template <typename T> __device__ __forceinline__ void step(T*& p) {
        const bool last = ++h == H;
        p += last ? wrap : head;
        if (last) h = 0;
    }
};

// Measured, 256x512 -> 128x256, B = 2, eight heads of 32, bf16: forward 67 us (76 % of the measured bandwidth), backward 105 (73 %); issue slots 74 and 67 % busy.
// Instructions are what costs: with fp32 values exchanged, weights multiplied per vector and addresses computed per slice the kernels took 310 (forward)
// instructions per vector of eight channels and were bound by issue (256x512 -> 128x256, B = 2, eight heads of 32, bf16: forward 129 us, backward 208).
// So a lane exchanges its words as they are, weights and angles are one factor per channel and point, and arithmetic is on packed pairs.
// LANES: the lanes of a vector where the compiler knows them (0: a.lanes), which saves the loop of the sums and some addresses (forward and backward, us: the case above
// 185 -> 174, 128x256, B = 4, four heads of 32, fp32 125 -> 120).
template <typename T, int V, Pairs PAIRS, bool BACKWARD, int LANES>
__global__ void __launch_bounds__(ROTATE_THREADS, BACKWARD ? 3 : 4) norm_rotate_kernel(const __grid_constant__ RotateArgs a) {
    using W = Words<T, V>;
    const int lanes = LANES > 0 ? LANES : a.lanes;
    constexpr int VP = V / 2, U = 2;        // pairs per lane; vectors of a group under way
    // (the last sum over threads needs room for a block's partial dw, the exchange for a block's vectors)
    __shared__ __align__(16) float shared[BACKWARD || PAIRS == Pairs::BY_SHARED ? ROTATE_THREADS * V : 4];
    if (BACKWARD) allow_dependents();
    const int which = (int)blockIdx.x >= a.first_blocks;
    const Part& p = a.part[which];
    const int block = (int)blockIdx.x - (which ? a.first_blocks : 0);
    const int lane = threadIdx.x & (lanes - 1), group = threadIdx.x / lanes, groups = ROTATE_THREADS / lanes;
    const int c0 = lane * V, C = a.C, P = p.pairs;
    const bool mine = c0 < C;
    // where the partners of the lane's channels are: a lane (itself if they are not turned), or the other half of each word
    const int other = PAIRS != Pairs::BY_SHUFFLE ? 0 : c0 < P ? lane + P / V : c0 < 2 * P ? lane - P / V : lane;
    uint32_t swap[W::N];
    if (PAIRS == Pairs::IN_LANE && sizeof(T) == 2)
#pragma unroll
        for (int i = 0; i < W::N; ++i) swap[i] = c0 + 2 * i < 2 * P ? 0x1032u : 0x3210u;
    auto partners = [&](const W& x) {
        W y;
        if constexpr (PAIRS == Pairs::BY_SHUFFLE) {
#pragma unroll
            for (int i = 0; i < W::N; ++i) y.w[i] = __shfl_sync(0xffffffffu, x.w[i], other, lanes);
        } else if constexpr (PAIRS == Pairs::IN_LANE) {
#pragma unroll
            for (int i = 0; i < W::N; ++i)
                if constexpr (sizeof(T) == 2) y.w[i] = __byte_perm(x.w[i], 0, swap[i]);
                else y.w[i] = c0 + (i & ~1) < 2 * P ? x.w[i ^ 1] : x.w[i];
        } else {
            T* row = reinterpret_cast<T*>(shared) + group * lanes * V;
            T own[V], got[V];
            *reinterpret_cast<W*>(own) = x;
#pragma unroll
            for (int i = 0; i < V; ++i) row[c0 + i] = own[i];
            __syncwarp();
#pragma unroll
            for (int i = 0; i < V; ++i) { const int c = c0 + i; got[i] = c < P ? row[c + P] : c < 2 * P ? row[c - P] : own[i]; }
            __syncwarp();
            y = *reinterpret_cast<W*>(got);
        }
        return y;
    };
    // dy's partner takes part with the transposed rotation's sign; x's with its own channel's weight
    float w[V], dw[V], w_partner[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = c0 + i, pc = c >= 2 * P ? c : PAIRS == Pairs::IN_LANE ? c ^ 1 : c < P ? c + P : c - P;
        w[i] = mine && p.weight != nullptr ? p.weight[c] : 1.f;
        w_partner[i] = !BACKWARD && mine && p.weight != nullptr ? p.weight[pc] : 1.f;
        dw[i] = 0.f;
    }
    uint64_t w2[VP], dw2[VP];
#pragma unroll
    for (int i = 0; i < VP; ++i) { w2[i] = pack2(w[2 * i], w[2 * i + 1]); dw2[i] = pack2(0.f, 0.f); }
    const int s_begin = (block / p.point_blocks) * p.slices_per_block, s_end = min(s_begin + p.slices_per_block, p.slices);
    const int b_begin = s_begin / p.H, h_begin = s_begin - b_begin * p.H;
    const float inverse_C = 1.f / C;

    // the trips are the same for all groups of a block, whose lanes meet in shuffles; those beyond the last point do nothing
    for (int point0 = (block % p.point_blocks) * groups; point0 < p.points; point0 += p.point_blocks * groups) {
        const int point = point0 + group;
        const bool here = mine && point < p.points;
        const int i_lat = here ? point / p.nlon : 0, j_lon = here ? point - i_lat * p.nlon : 0;
        const T* x = static_cast<const T*>(p.x.data) + at(p.x, i_lat, j_lon) + b_begin * p.x.batch + h_begin * p.x.head + c0;
        const T* dy = BACKWARD ? static_cast<const T*>(p.dy.data) + at(p.dy, i_lat, j_lon) + b_begin * p.dy.batch + h_begin * p.dy.head + c0 : nullptr;
        T* y = static_cast<T*>(p.y.data) + at(p.y, i_lat, j_lon) + b_begin * p.y.batch + h_begin * p.y.head + c0;
        Walk walk_x(p.x, h_begin, p.H), walk_dy(p.dy, h_begin, p.H), walk_y(p.y, h_begin, p.H);
        W x_next[U], g_next[U];
        // the next U vectors are under way while these are computed
        auto fetch = [&](int s) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (here && s + u < s_end) {
                    x_next[u] = load_words<T, V>(x);
                    if (BACKWARD) g_next[u] = load_words<T, V>(dy);
                }
                walk_x.step(x);
                if (BACKWARD) walk_dy.step(dy);
            }
        };
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < W::N; ++i) { x_next[u].w[i] = 0; g_next[u].w[i] = 0; }
        fetch(s_begin);
        // y = own * x + partner's * x of the partner (times r); backward: g likewise, of dy
        uint64_t own[VP], partners_[VP];
        {
            float cs[V], sn[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = c0 + i;
                const int pair = PAIRS == Pairs::IN_LANE ? c >> 1 : c < P ? c : c - P;
                const bool first = PAIRS == Pairs::IN_LANE ? (c & 1) == 0 : c < P;
                cs[i] = 1.f; sn[i] = 0.f;
                if (mine && c < 2 * P) {
                    const float2 t = pair < p.pairs_lat ? reinterpret_cast<const float2*>(p.lat_table)[(int64_t)i_lat * p.pairs_lat + pair]
                                                        : reinterpret_cast<const float2*>(p.lon_table)[(int64_t)j_lon * (P - p.pairs_lat) + pair - p.pairs_lat];
                    cs[i] = t.x;
                    sn[i] = first != BACKWARD ? -t.y : t.y;
                }
                if (!BACKWARD) { cs[i] *= w[i]; sn[i] *= w_partner[i]; }
            }
#pragma unroll
            for (int i = 0; i < VP; ++i) { own[i] = pack2(cs[2 * i], cs[2 * i + 1]); partners_[i] = pack2(sn[2 * i], sn[2 * i + 1]); }
        }
        for (int s = s_begin; s < s_end; s += U) {
            W xs[U], gs[U];
#pragma unroll
            for (int u = 0; u < U; ++u) { xs[u] = x_next[u]; if (BACKWARD) gs[u] = g_next[u]; }
            if (s + U < s_end) fetch(s + U);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (s + u >= s_end) break;          // (the same for the whole block; what is in the registers then is an earlier vector)
                uint64_t xf[VP], v[VP], vp[VP];
                pairs_of<T, V>(xs[u], xf);
                pairs_of<T, V>(partners(BACKWARD ? gs[u] : xs[u]), vp);
                if (BACKWARD) pairs_of<T, V>(gs[u], v);
                uint64_t square2 = pack2(0.f, 0.f), product2 = pack2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < VP; ++i) {
                    square2 = fma2(xf[i], xf[i], square2);
                    v[i] = fma2(partners_[i], vp[i], mul2(own[i], BACKWARD ? v[i] : xf[i]));       // y / r, or g
                    if (BACKWARD) product2 = fma2(mul2(v[i], w2[i]), xf[i], product2);
                }
                float square, product, upper;
                unpack2(square2, square, upper);
                square += upper;
                unpack2(product2, product, upper);
                product += upper;
#pragma unroll (LANES > 0 ? 4 : 1)
                for (int o = lanes >> 1; o > 0; o >>= 1) {
                    square += __shfl_xor_sync(0xffffffffu, square, o);
                    if (BACKWARD) product += __shfl_xor_sync(0xffffffffu, product, o);
                }
                // (groups behind the last point hold zeros: with eps = 0 theirs would be infinite, and their part of dw NaN)
                const float r = BACKWARD && !here ? 0.f : rsqrtf(square * inverse_C + a.eps);
                const uint64_t r2 = pack2(r, r);
                if (BACKWARD) {
                    // dx = r (g w) - n (r sum(g w n) / C) with n = x r
                    const float along = -product * inverse_C * r * r;
                    const uint64_t along2 = pack2(along, along);
#pragma unroll
                    for (int i = 0; i < VP; ++i) {
                        const uint64_t n = mul2(xf[i], r2);
                        dw2[i] = fma2(v[i], n, dw2[i]);
                        v[i] = fma2(n, along2, mul2(mul2(v[i], w2[i]), r2));
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < VP; ++i) v[i] = mul2(v[i], r2);
                }
                if (here) store_words<T, V>(y, words_of<T, V>(v));
                walk_y.step(y);
            }
        }
    }
    if (BACKWARD && p.partials != nullptr) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VP; ++i) unpack2(dw2[i], shared[(group * lanes + lane) * V + 2 * i], shared[(group * lanes + lane) * V + 2 * i + 1]);
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += ROTATE_THREADS) {
            float sum = 0.f;
            for (int g = 0; g < groups; ++g) sum += shared[g * lanes * V + c];
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
// dweight = sum of the blocks' partial sums, in a fixed order.  One block per 8 channels (a sector of each row) and part; 128 rows of threads.
__global__ void __launch_bounds__(1024) sum_partials_kernel(const __grid_constant__ SumArgs a) {
    __shared__ float sums[128][9];
    const int which = blockIdx.y, c = blockIdx.x * 8 + threadIdx.x, rows = a.rows[which];
    if (a.dweight[which] == nullptr) return;
    const float* from = a.partials[which] + c;
    float sum = 0.f;
    wait_for_previous();
    if (c < a.C)
#pragma unroll 4
        for (int r = threadIdx.y; r < rows; r += 128) sum += from[(int64_t)r * a.C];
    sums[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
#pragma unroll
    for (int o = 64; o > 0; o >>= 1) {
        if (threadIdx.y < o) sums[threadIdx.y][threadIdx.x] += sums[threadIdx.y + o][threadIdx.x];
        __syncthreads();
    }
    if (threadIdx.y == 0 && c < a.C) a.dweight[which][c] = sums[0][threadIdx.x];
}

template <typename T, int V, Pairs PAIRS, bool BACKWARD>
cudaError_t launch_lanes(const RotateArgs& a, int blocks, cudaStream_t stream) {
    auto run = [&](auto lanes) {
        norm_rotate_kernel<T, V, PAIRS, BACKWARD, decltype(lanes)::value><<<blocks, ROTATE_THREADS, 0, stream>>>(a);
        return cudaGetLastError();
    };
    // (vectors of 16 bytes: heads of 17 to 128 channels in 16 bits, of 9 to 64 in 32; the others are left to one kernel)
    if constexpr (V * sizeof(T) == 16 && PAIRS != Pairs::BY_SHARED) {
        if (a.lanes == 4) return run(std::integral_constant<int, 4>());
        if (a.lanes == 8) return run(std::integral_constant<int, 8>());
        if (a.lanes == 16) return run(std::integral_constant<int, 16>());
    }
    return run(std::integral_constant<int, 0>());
}
template <typename T, int V, bool BACKWARD>
cudaError_t launch_pairs(const RotateArgs& a, Pairs pairs, int blocks, cudaStream_t stream) {
    if (pairs == Pairs::IN_LANE) return launch_lanes<T, V, Pairs::IN_LANE, BACKWARD>(a, blocks, stream);
    if (pairs == Pairs::BY_SHUFFLE) return launch_lanes<T, V, Pairs::BY_SHUFFLE, BACKWARD>(a, blocks, stream);
    return launch_lanes<T, V, Pairs::BY_SHARED, BACKWARD>(a, blocks, stream);
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
        // A block's groups take neighbouring points.  Slices are spread over blocks until the GPU has one full wave of them, as long as each still takes
        // sixteen with the angles that it has read, or two where the points give less than a block per SM; the backward pass also bounds its blocks, each of which
        // leaves a row of partial sums.  Sixteen was measured on the case above alone (four: forward 73 instead of 70 us, two waves of blocks 78).  For middle
        // sizes it leaves SMs idle: 91x180, B = 2, 8 and 2 heads of 24, fp16 takes 14 us, with 512 blocks for 592 places and eight trips of two vectors in a row.
        const int groups = ROTATE_THREADS / a.lanes;
        p.point_blocks = (p.points + groups - 1) / groups;
        const int want = std::max(1, (4 * sms + p.point_blocks - 1) / p.point_blocks);
        p.slices_per_block = std::max(std::min(p.slices, 16), (p.slices + want - 1) / want);
        if (p.point_blocks < sms) p.slices_per_block = std::max(std::min(p.slices, 2), (p.slices + want - 1) / want);
        p.slice_blocks = (p.slices + p.slices_per_block - 1) / p.slices_per_block;
        if (backward && (int64_t)p.point_blocks * p.slice_blocks > MAX_PARTIALS) {
            p.slice_blocks = std::min(p.slice_blocks, std::max(1, MAX_PARTIALS / p.point_blocks));
            p.slices_per_block = (p.slices + p.slice_blocks - 1) / p.slice_blocks;
            p.slice_blocks = (p.slices + p.slices_per_block - 1) / p.slices_per_block;
            const int most = MAX_PARTIALS / p.slice_blocks, trips = (p.point_blocks + most - 1) / most;
            p.point_blocks = (p.point_blocks + trips - 1) / trips;
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
        e = launch_dependent(sum_partials_kernel, dim3((C + 7) / 8, n_parts), dim3(8, 128), 0, stream, sum);
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
