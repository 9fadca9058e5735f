// Softmax attention over all points with a logarithmic weight per point, 16-bit tensors: forward pass, its form for few queries, and the
// backward pass that recomputes the probabilities.
//
//   s_ij = scale q_i.k_j + w_j,  p_ij = exp(s_ij - lse_i),  out_i = sum_j p_ij v_j,  lse_i = log sum_j exp(s_ij)
//   t_ij = dout_i.v_j,  D_i = dout_i.out_i,  ds_ij = p_ij (t_ij - D_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij dout_i
//
// These are the kernels for any size, on mma.sync (m16n8k16): a warp owns 16 rows, scores stay in registers and become the next product's
// operand there.  Products are accumulated in 32 bits, the softmax and all statistics are in 32 bits.  p and ds are operands of
// the second products in two 16-bit parts (one station over 361x720, B = 2, 8 and 2 heads of 64, bf16: 53.3 us and a relative error of 0.0017, that of rounding the result;
// with p rounded once 52.9 us and 0.0020).
//
// A key head serves G query heads: their rows are stacked, so that the head's keys are read once for all of them, and so that its
// gradients are summed within one block.  Few rows: a tile of 16 rows, the block's four warps sharing each 64 keys, and the keys split
// over blocks whose partial results a second kernel joins.
//
// A point whose weight leaves it out is read as zeros, whatever it holds, and has a weight of exactly zero.  A row without any point has
// out = 0, lse = -infinity, and no gradient.  Both hold for queries and gradients of infinities and NaN, too, whose products with those zeros are NaN.
#include <algorithm>

#include "sna_attend.cuh"

namespace sna {
namespace attend {
namespace {

constexpr int BN = 64;              // keys (or queries) per streamed block
constexpr int WARPS = 4, THREADS = 32 * WARPS;

__device__ __forceinline__ uint32_t s32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_group() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T> __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <typename T> __device__ __forceinline__ uint32_t pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t pack<__half>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// The A operand of a second product from 16 x 16 numbers in a product's layout (two 16 x 8 accumulators), rounded to 16 bits, and what rounding leaves: with
// both, p and ds count with twice the digits.  These kernels take the small problems, whose time is not the tensor cores'; of the tcgen05 kernels
// the forward one rounds once, and so does the backward one except for narrow heads and small problems (in_two_parts).
template <typename T>
__device__ __forceinline__ void operands(const float (&x)[4], const float (&y)[4], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
    const float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        hi[i] = pack<T>(v[2 * i], v[2 * i + 1]);
        float a, b;
        unpack2(pair_of<T>(hi[i]), a, b);
        lo[i] = pack<T>(v[2 * i] - a, v[2 * i + 1] - b);
    }
}

// A tile in shared memory: rows of CP 16-bit channels in pieces of 16 bytes, which are permuted within a row so that the eight rows of an
// 8x8 matrix meet different banks.
template <int CP> __device__ __forceinline__ uint32_t piece(int row, int c) {
    constexpr int CH = CP / 8;
    return (uint32_t)(row * CP * 2 + ((c ^ (CH >= 8 ? row & 7 : (row >> 1) & 3)) << 4));
}
// The A operand (16 rows x 16 channels) of rows row0 .. row0 + 15 at channel step ks
template <int CP> __device__ __forceinline__ void load_a(uint32_t (&a)[4], uint32_t tile, int row0, int ks, int lane) {
    ldsm(a, tile + piece<CP>(row0 + (lane & 15), ks * 2 + (lane >> 4)));
}
// B operands of 16 rows n0 .. n0 + 15 (as columns of the product) at channel step ks: b[0], b[1] for the first eight, b[2], b[3]
template <int CP> __device__ __forceinline__ void load_b(uint32_t (&b)[4], uint32_t tile, int n0, int ks, int lane) {
    ldsm(b, tile + piece<CP>(n0 + (lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)));
}
// B operands for a sum over rows k0 .. k0 + 15 of 16 channels from 16 * n
template <int CP> __device__ __forceinline__ void load_bt(uint32_t (&b)[4], uint32_t tile, int k0, int n, int lane) {
    ldsm_t(b, tile + piece<CP>(k0 + (lane & 7) + (((lane >> 3) & 1) << 3), n * 2 + (lane >> 4)));
}

// rows [first, first + R) of a head's points (stride `point`); a row that is not there, or for which take(row in tile) is false, is zero.
// A thread's pieces lie RP rows apart, which is a multiple of the permutation's period: one address each way, and steps.  take also sees to rows
// behind the last point.
template <int CP, int R, typename T, typename Take>
__device__ __forceinline__ void load_rows(uint32_t tile, const T* head, int64_t point, int first, int C, Take take) {
    constexpr int CH = CP / 8, RP = THREADS / CH;
    static_assert(RP % 8 == 0 && R % RP == 0, "steps of whole periods");
    const int r0 = threadIdx.x / CH, c = threadIdx.x - r0 * CH;
    const T* src = head + (first + r0) * point + c * 8;
    const uint32_t dst = tile + piece<CP>(r0, c);
    const bool channel = c * 8 < C;
#pragma unroll
    for (int i = 0; i < R / RP; ++i) {
        const bool there = channel && take(r0 + i * RP);
        copy16(dst + i * RP * CP * 2, there ? src : head, there);
        src += RP * point;
    }
}
// the same for the stacked rows of the query heads of a group: row = head in the group * Nq + query
template <int CP, typename T>
__device__ __forceinline__ void load_stacked(uint32_t tile, const T* group, int64_t head, int64_t point, int first, int rows, int Nq, int R, int C) {
    constexpr int CH = CP / 8;
    for (int e = threadIdx.x; e < R * CH; e += THREADS) {
        const int r = e / CH, c = e - r * CH, row = first + r;
        const bool there = row < rows && c * 8 < C;
        const int g = there ? row / Nq : 0;
        copy16(tile + piece<CP>(r, c), there ? group + g * head + (int64_t)(row - g * Nq) * point + c * 8 : group, there);
    }
}

// log2 of a point's weight, -infinity if it is left out
__device__ __forceinline__ float weight2(const float* weights, int n) {
    if (weights == nullptr) return 0.f;
    const float w = weights[n];
    return w <= EXCLUDED ? -INFINITY : w * LOG2E;
}

// ---- forward ---------------------------------------------------------------------------------------------------------------

// One value of out, and what its rounding leaves.
template <typename T>
__device__ __forceinline__ void store_out(const Problem& p, int64_t b, int64_t h, int64_t n, int c, float x) {
    const T rounded = from_float<T>(x);
    static_cast<T*>(p.out.data)[b * p.out.batch + h * p.out.head + n * p.out.point + c] = rounded;
    if (p.rest.data != nullptr) static_cast<T*>(p.rest.data)[b * p.rest.batch + h * p.rest.head + n * p.rest.point + c] = from_float<T>(x - to_float(rounded));
}

// Stages of (K, V).  One station over 361x720, B = 2, 8 and 2 heads of 64, bf16, four blocks per SM, with the join: 53 us (these with p rounded once); three stages 56, four 68; five blocks per SM
// 54, six 61 (with fewer registers each).  A warp that loads and waits for its own keys alone gained nothing.
constexpr int FORWARD_STAGES = 2;
template <int CP, int WM> constexpr int forward_smem() { return WM * 16 * CP * 2 + FORWARD_STAGES * 2 * BN * CP * 2; }

// WM warps along the rows, WK = 4 / WM along the keys of a block.  partials: null, or sums [splits][rows][C] (first, so that vectors stay aligned) and statistics
// [splits][rows].
template <typename T, int CP, int WM>
__global__ void __launch_bounds__(THREADS, WM == 1 && CP <= 64 ? 4 : 1) attend_forward_kernel(const __grid_constant__ Problem p, int tiles, int splits, float* partials) {
    constexpr int STAGES = FORWARD_STAGES, WK = WARPS / WM, BM = 16 * WM, KW = BN / WK, NT = KW / 8, CN = CP / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(16) float bias[8][BN];
    const uint32_t tq = s32(smem), tkv = tq + BM * CP * 2;      // stages of (K, V)
    allow_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wm = warp % WM, wk = warp / WM;
    const int split = blockIdx.x % splits, rest = blockIdx.x / splits, tile = rest % tiles, bh = rest / tiles;
    const int b = bh / p.Hk, hk = bh - b * p.Hk;
    const int rows = p.G * p.Nq, row0 = tile * BM;
    const T* kh = static_cast<const T*>(p.k.data) + b * p.k.batch + hk * p.k.head;
    const T* vh = static_cast<const T*>(p.v.data) + b * p.v.batch + hk * p.v.head;
    const float* weights = p.log_weights == nullptr ? nullptr : p.log_weights + b * p.log_weights_batch;
    const int blocks = (p.Nk + BN - 1) / BN;
    const int first = (int)((int64_t)blocks * split / splits), last = (int)((int64_t)blocks * (split + 1) / splits);

    // Weights come by asynchronous copies 2 STAGES blocks ahead, and are made ready (log2, -infinity for points left out) STAGES ahead, in place: the loads of a
    // block's keys and values go by them.  (Read into a register one step ahead, they were what the steps waited for: one station over 361x720, B = 2, 2 key heads
    // of 32, bf16: 47 us with weights, 35 without.)
    auto ready = [&](int j, float raw) { return j >= last || j * BN + tid >= p.Nk ? -INFINITY : weights == nullptr ? 0.f : raw <= EXCLUDED ? -INFINITY : raw * LOG2E; };
    auto copy_bias = [&](int j) {
        if (weights != nullptr && tid < BN && j < last && j * BN + tid < p.Nk) copy4(s32(&bias[j & 7][tid]), weights + j * BN + tid);
    };
    auto ready_bias = [&](int j) {
        if (tid < BN) bias[j & 7][tid] = ready(j, bias[j & 7][tid]);
    };
    auto load_block = [&](int j) {
        if (j < last) {
            const uint32_t stage = tkv + ((j - first) % STAGES) * 2 * BN * CP * 2;
            auto take = [&](int r) { return bias[j & 7][r] != -INFINITY; };
            load_rows<CP, BN>(stage, kh, p.k.point, j * BN, p.C, take);
            load_rows<CP, BN>(stage + BN * CP * 2, vh, p.v.point, j * BN, p.C, take);
        }
        commit();
    };
    load_stacked<CP>(tq, static_cast<const T*>(p.q.data) + b * p.q.batch + (int64_t)hk * p.G * p.q.head, p.q.head, p.q.point, row0, rows, p.Nq, BM, p.C);
#pragma unroll
    for (int i = 0; i < 2 * STAGES; ++i)
        if (tid < BN) {
            const int j = first + i, n = j * BN + tid;
            const float raw = weights != nullptr && j < last && n < p.Nk ? weights[n] : 0.f;
            bias[j & 7][tid] = i < STAGES ? ready(j, raw) : raw;
        }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) load_block(first + i);

    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[CN][4];
#pragma unroll
    for (int n = 0; n < CN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][i] = 0.f;

    uint32_t q[WM == 1 ? CP / 16 : 1][4];        // few rows: the queries' operands stay in registers
    if (WM == 1) {
        wait_group<STAGES - 2>();
        __syncthreads();
#pragma unroll
        for (int ks = 0; ks < CP / 16; ++ks) load_a<CP>(q[WM == 1 ? ks : 0], tq, 0, ks, lane);
    }
    for (int j = first; j < last; ++j) {
        ready_bias(j + STAGES);
        copy_bias(j + 2 * STAGES);
        load_block(j + STAGES - 1);
        wait_group<STAGES - 1>();
        __syncthreads();
        const uint32_t tk = tkv + ((j - first) % STAGES) * 2 * BN * CP * 2, tv = tk + BN * CP * 2;
        const int key0 = wk * KW;
        float s[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[n][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < CP / 16; ++ks) {
            uint32_t (&a)[4] = q[WM == 1 ? ks : 0];
            if (WM != 1) load_a<CP>(a, tq, wm * 16, ks, lane);
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                uint32_t kb[4];
                load_b<CP>(kb, tk, key0 + n * 8, ks, lane);
                mma<T>(s[n], a, kb[0], kb[1]);
                mma<T>(s[n + 1], a, kb[2], kb[3]);
            }
        }
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float2 w = *reinterpret_cast<const float2*>(&bias[j & 7][key0 + n * 8 + (lane & 3) * 2]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][i] = fmaf(s[n][i], p.scale_log2, (i & 1) ? w.y : w.x);
                top[i >> 1] = fmaxf(top[i >> 1], s[n][i]);
            }
        }
        float base[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
            const float now = fmaxf(m[r], top[r]);
            base[r] = now == -INFINITY ? 0.f : now;                 // (no point so far: every weight is exp2(-infinity))
            if (__any_sync(0xffffffffu, now != m[r])) {         // (a new maximum gets rare)
                const float correction = ex2(m[r] - base[r]);
                l[r] *= correction;
#pragma unroll
                for (int n = 0; n < CN; ++n) { o[n][2 * r] *= correction; o[n][2 * r + 1] *= correction; }
            }
            m[r] = now;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][i] = ex2(s[n][i] - base[i >> 1] + SHIFT<T>);
                l[i >> 1] += s[n][i];
            }
#pragma unroll
        for (int ks = 0; ks < KW / 16; ++ks) {
            uint32_t a[4], a_lo[4];
            operands<T>(s[2 * ks], s[2 * ks + 1], a, a_lo);
#pragma unroll
            for (int n = 0; n < CN; n += 2) {
                uint32_t vb[4];
                load_bt<CP>(vb, tv, key0 + ks * 16, n / 2, lane);
                mma<T>(o[n], a_lo, vb[0], vb[1]);
                mma<T>(o[n + 1], a_lo, vb[2], vb[3]);
                mma<T>(o[n], a, vb[0], vb[1]);
                mma<T>(o[n + 1], a, vb[2], vb[3]);
            }
        }
        __syncthreads();        // before the stage is overwritten
    }
    wait_group<0>();
    // A query of infinities or NaN makes scores NaN against the zeros of points left out, too: with those alone its row is one without points.
    bool nothing = false;
    if (weights != nullptr && __syncthreads_or(l[0] != l[0] || l[1] != l[1])) {
        bool present = false;
        for (int n = first * BN + tid; n < p.Nk && n < last * BN; n += THREADS) present |= !(weights[n] <= EXCLUDED);
        nothing = __syncthreads_or(present) == 0;
    }
    if (nothing) {
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
#pragma unroll
        for (int n = 0; n < CN; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    }
    if constexpr (WK > 1) {
        // the warps' sums of the same rows are joined in the stages' memory: [warp][row][CP + 2]
        __syncthreads();
        float* join = reinterpret_cast<float*>(smem + BM * CP * 2);
        constexpr int PITCH = CP + 4;
        static_assert(WARPS * 16 * PITCH * 4 <= 4 * BN * CP * 2, "the join fits");
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float* mine = join + (warp * 16 + (lane >> 2) + 8 * r) * PITCH;
            if ((lane & 3) == 0) { mine[CP] = m[r]; mine[CP + 1] = l[r]; }
#pragma unroll
            for (int n = 0; n < CN; ++n) *reinterpret_cast<float2*>(mine + n * 8 + (lane & 3) * 2) = make_float2(o[n][2 * r], o[n][2 * r + 1]);
        }
        __syncthreads();
        // warp w joins rows 4 w .. 4 w + 3
        for (int r = warp * 4; r < warp * 4 + 4; ++r) {
            float top = -INFINITY, total = 0.f;
            for (int w = 0; w < WARPS; ++w) top = fmaxf(top, join[(w * 16 + r) * PITCH + CP]);
            const float base = top == -INFINITY ? 0.f : top;
            float factor[WARPS];
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                factor[w] = ex2(join[(w * 16 + r) * PITCH + CP] - base);
                total += factor[w] * join[(w * 16 + r) * PITCH + CP + 1];
            }
            const int row = row0 + r;
            if (row >= rows) continue;
            const int g = row / p.Nq;
            const int64_t at = ((int64_t)b * p.Hq + hk * p.G + g) * p.Nq + (row - g * p.Nq);
            const float inverse = total == 0.f ? 0.f : 1.f / total;
            const float lse2 = total == 0.f ? -INFINITY : top + log2f(total) - SHIFT<T>;
            for (int c = lane; c < p.C; c += 32) {
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < WARPS; ++w) sum += factor[w] * join[(w * 16 + r) * PITCH + c];
                if (partials != nullptr) partials[((int64_t)split * rows_of(p) + at) * p.C + c] = sum * inverse;
                else store_out<T>(p, b, hk * p.G + g, row - g * p.Nq, c, sum * inverse);
            }
            if (lane == 0) {
                if (partials != nullptr) partials[splits * rows_of(p) * p.C + split * rows_of(p) + at] = lse2;
                else if (p.lse != nullptr) p.lse[at] = lse2 * LN2;
            }
        }
    } else {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = row0 + wm * 16 + (lane >> 2) + 8 * r;
            if (row >= rows) continue;
            const int g = row / p.Nq;
            const int64_t at = ((int64_t)b * p.Hq + hk * p.G + g) * p.Nq + (row - g * p.Nq);
            const float inverse = l[r] == 0.f ? 0.f : 1.f / l[r];
            const float lse2 = l[r] == 0.f ? -INFINITY : m[r] + log2f(l[r]) - SHIFT<T>;
            T* out = static_cast<T*>(p.out.data) + b * p.out.batch + (int64_t)(hk * p.G + g) * p.out.head + (int64_t)(row - g * p.Nq) * p.out.point;
#pragma unroll
            for (int n = 0; n < CN; ++n) {
                const int c = n * 8 + (lane & 3) * 2;
                if (c >= p.C) continue;
                const float x = o[n][2 * r] * inverse, y = o[n][2 * r + 1] * inverse;
                if (partials != nullptr) *reinterpret_cast<float2*>(partials + ((int64_t)split * rows_of(p) + at) * p.C + c) = make_float2(x, y);
                else {
                    const uint32_t word = pack<T>(x, y);
                    *reinterpret_cast<uint32_t*>(out + c) = word;
                    if (p.rest.data != nullptr) {
                        float hi_x, hi_y;
                        unpack2(pair_of<T>(word), hi_x, hi_y);
                        T* rest = static_cast<T*>(p.rest.data) + b * p.rest.batch + (int64_t)(hk * p.G + g) * p.rest.head + (int64_t)(row - g * p.Nq) * p.rest.point;
                        *reinterpret_cast<uint32_t*>(rest + c) = pack<T>(x - hi_x, y - hi_y);
                    }
                }
            }
            if ((lane & 3) == 0) {
                if (partials != nullptr) partials[splits * rows_of(p) * p.C + split * rows_of(p) + at] = lse2;
                else if (p.lse != nullptr) p.lse[at] = lse2 * LN2;
            }
        }
    }
}

// Joins the splits' results of a row: out = sum_s 2^(lse2_s - lse2) out_s, the sum taken in a fixed order.
// Few rows and many splits: a block of eight warps per row, warp w takes the splits w, w + 8, ...  Otherwise a warp per row.
constexpr int JOIN_WARPS = 8;
template <typename T, bool BLOCK_PER_ROW>
__global__ void __launch_bounds__(32 * JOIN_WARPS) attend_join_kernel(const __grid_constant__ Problem p, int splits, const float* partials) {
    __shared__ float sums[BLOCK_PER_ROW ? JOIN_WARPS : 1][128];
    __shared__ float totals[JOIN_WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t rows = rows_of(p), at = BLOCK_PER_ROW ? blockIdx.x : (int64_t)blockIdx.x * JOIN_WARPS + warp;
    if (at >= rows) return;         // (whole warps; whole blocks where they meet)
    wait_for_previous();
    const float* statistics = partials + splits * rows * p.C;
    float top = -INFINITY;
    for (int s = lane; s < splits; s += 32) top = fmaxf(top, statistics[s * rows + at]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float base = top == -INFINITY ? 0.f : top;
    float sum[4] = {0.f, 0.f, 0.f, 0.f}, total = 0.f;
#pragma unroll 4
    for (int s = BLOCK_PER_ROW ? warp : 0; s < splits; s += BLOCK_PER_ROW ? JOIN_WARPS : 1) {
        const float w = ex2(statistics[s * rows + at] - base);
        total += w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < p.C) sum[i] = fmaf(w, partials[(s * rows + at) * p.C + lane + 32 * i], sum[i]);
    }
    if constexpr (BLOCK_PER_ROW) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[warp][lane + 32 * i] = sum[i];
        if (lane == 0) totals[warp] = total;
        __syncthreads();
        if (warp != 0) return;
        total = 0.f;
#pragma unroll
        for (int w = 0; w < JOIN_WARPS; ++w) total += totals[w];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum[i] = 0.f;
#pragma unroll
            for (int w = 0; w < JOIN_WARPS; ++w) sum[i] += sums[w][lane + 32 * i];
        }
    }
    const int n = (int)(at % p.Nq);
    const int64_t bh = at / p.Nq, b = bh / p.Hq, h = bh - b * p.Hq;
    const float inverse = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 32 * i < p.C) store_out<T>(p, b, h, n, lane + 32 * i, sum[i] * inverse);
    if (lane == 0 && p.lse != nullptr) p.lse[at] = total == 0.f ? -INFINITY : (top + log2f(total)) * LN2;
}

// ---- points that take part ----------------------------------------------------------------------------------------------------

// A block of 256 threads, for 256 points of one batch and key head; the blocks of the first head write the lists.  Backward (s is there): also the weights that the
// dq kernel adds to S, and the gradients of the points left out.
__device__ __forceinline__ void select_points(const Problem& p, const Selection& sel, const Stats* s, int64_t block) {
    constexpr int N = SELECT_POINTS, NW = N / 32;
    __shared__ int sums[NW][3];
    __shared__ int list[N];             // taken points from the front, left-out ones from the back
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cuts = (p.Nk + N - 1) / N;
    const int64_t bh = block / cuts, b = bh / p.Hk, hk = bh - b * p.Hk;
    const int first = (int)(block - bh * cuts) * N, n = first + tid, here = min(N, p.Nk - first);
    const float* weights = p.log_weights + b * p.log_weights_batch;
    int before = 0, total = 0;
#pragma unroll 16
    for (int i = tid; i < p.Nk; i += N) {
        const int take = !(weights[i] <= EXCLUDED);
        total += take;
        before += i < first ? take : 0;
    }
    total = __reduce_add_sync(0xffffffffu, total);
    before = __reduce_add_sync(0xffffffffu, before);
    const float weight = n < p.Nk ? weights[n] : -INFINITY;
    const bool take = n < p.Nk && !(weight <= EXCLUDED);
    const uint32_t takes = __ballot_sync(0xffffffffu, take);
    if (lane == 0) { sums[warp][0] = total; sums[warp][1] = before; sums[warp][2] = __popc(takes); }
    __syncthreads();
    int rank = __popc(takes & ((1u << lane) - 1u)), m = 0;
    total = before = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        total += sums[w][0];
        before += sums[w][1];
        rank += w < warp ? sums[w][2] : 0;
        m += sums[w][2];
    }
    const bool apart = total <= p.Nk - p.Nk / 16;
    const int per_row = (p.Nk + STATS_BLOCK - 1) / STATS_BLOCK;
    if (hk == 0) {
        if (block == bh * cuts && tid == 0) sel.taken[b] = apart ? total : p.Nk;
        const int at = apart ? before + rank : n;
        if (apart && take) {
            sel.index[b * p.Nk + at] = n;
            sel.weights[b * p.Nk + at] = weight;
        }
        if (s != nullptr) {
            uint4* extra = s->weights + b * per_row * STATS_BLOCK;
            const uint2 parts = take ? extra_parts(weight / p.scale) : make_uint2(EXTRA_OUT, 0);
            if (apart ? take : n < per_row * STATS_BLOCK) extra[at] = make_uint4(parts.x, parts.y, 0, 0);
            if (!apart && lane == 0 && n < per_row * STATS_BLOCK)
                reinterpret_cast<uint32_t*>(s->gone + b * per_row)[n >> 5] = ~takes & (p.Nk - n >= 32 ? ~0u : p.Nk > n ? (1u << (p.Nk - n)) - 1u : 0u);
            if (apart && first + N >= p.Nk && total + tid < (total + STATS_BLOCK - 1) / STATS_BLOCK * STATS_BLOCK) extra[total + tid] = make_uint4(EXTRA_OUT, 0, 0, 0);
        }
    }
    if (!apart) return;
    if (n < p.Nk) list[take ? rank : here - 1 - (tid - rank)] = n;
    __syncthreads();
    const int chunks = p.C / 8;
    uint4 *k_to = static_cast<uint4*>(sel.k) + bh * p.Nk * chunks, *v_to = static_cast<uint4*>(sel.v) + bh * p.Nk * chunks;
    auto row = [&](const View& v, int r) { return reinterpret_cast<uint4*>(static_cast<uint16_t*>(v.data) + b * v.batch + hk * v.head + r * v.point); };
    for (int e = tid; e < m * chunks; e += N) {
        const int r = e / chunks, c = e - r * chunks;
        k_to[(before + r) * (int64_t)chunks + c] = row(p.k, list[r])[c];
        v_to[(before + r) * (int64_t)chunks + c] = row(p.v, list[r])[c];
    }
    if (s != nullptr)
        for (int e = tid; e < (here - m) * chunks; e += N) {
            const int r = e / chunks, c = e - r * chunks;
            row(p.dk, list[m + r])[c] = row(p.dv, list[m + r])[c] = make_uint4(0, 0, 0, 0);
        }
    if (first + N >= p.Nk) {
        const int end = min(p.Nk, (total + 127) / 128 * 128);
        for (int e = tid; e < (end - total) * chunks; e += N) k_to[total * (int64_t)chunks + e] = v_to[total * (int64_t)chunks + e] = make_uint4(0, 0, 0, 0);
    }
}
__global__ void __launch_bounds__(SELECT_POINTS) attend_select_kernel(const __grid_constant__ Problem p, const __grid_constant__ Selection sel) {
    allow_dependents();
    select_points(p, sel, nullptr, blockIdx.x);
}

// ---- backward: statistics -----------------------------------------------------------------------------------------------------

// Per query: D = dout . out, log2 of the sum of weights, and both as the extra rows that the tcgen05 dk/dv kernel copies.  float16: also the largest norm
// of a row of dout and of v per key head, which bound |t - D| <= 2 |dout| |v| (the last blocks take v's rows); a maximum does not depend on the
// order of its atomics, of which there is one per block (one per row took ten times as long as the rest).  A block takes 64 points of one head,
// four lanes each.  The first blocks prepare the points' weights for the tcgen05 dq kernel, or select them.
template <typename T>
__global__ void __launch_bounds__(256) attend_statistics_kernel(const __grid_constant__ Problem p, const __grid_constant__ Stats s, const __grid_constant__ Selection sel, int64_t query_blocks,
                                                                int64_t weight_blocks) {
    constexpr bool SCALED = SHIFT<T> != 0.f;
    __shared__ uint32_t most;
    allow_dependents();
    const int part = threadIdx.x & 3, place = threadIdx.x >> 2;
    if (blockIdx.x < weight_blocks) {
        if (sel.taken != nullptr) {
            select_points(p, sel, &s, blockIdx.x);
            return;
        }
        // one thread per point: its weight in parts, and who is left out
        const int per_row = (p.Nk + STATS_BLOCK - 1) / STATS_BLOCK, row = blockIdx.x / per_row, first = (blockIdx.x - row * per_row) * STATS_BLOCK;
        if (threadIdx.x >= STATS_BLOCK) return;
        const int n = first + threadIdx.x;
        const float weight = n < p.Nk ? p.log_weights[row * p.log_weights_batch + n] : -INFINITY;
        const bool out = weight <= EXCLUDED;
        const uint2 parts = out ? make_uint2(EXTRA_OUT, 0) : extra_parts(weight / p.scale);
        s.weights[(int64_t)blockIdx.x * STATS_BLOCK + threadIdx.x] = make_uint4(parts.x, parts.y, 0, 0);
        const uint32_t gone = __ballot_sync(0xffffffffu, out && n < p.Nk);
        if ((threadIdx.x & 31) == 0) reinterpret_cast<uint32_t*>(s.gone)[(int64_t)blockIdx.x * 2 + (threadIdx.x >> 5)] = gone;
        return;
    }
    const int64_t index = (int64_t)blockIdx.x - weight_blocks;
    const bool queries = index < query_blocks;
    const int64_t block = index - (queries ? 0 : query_blocks);
    const int N = queries ? p.Nq : p.Nk, H = queries ? p.Hq : p.Hk, per_head = (N + STATS_BLOCK - 1) / STATS_BLOCK;
    const int64_t bh = block / per_head, b = bh / H, h = bh - b * H;
    const int n = (int)(block - bh * per_head) * STATS_BLOCK + place;
    const bool there = n < N && (queries || p.log_weights == nullptr || !(p.log_weights[b * p.log_weights_batch + n] <= EXCLUDED));
    float square = 0.f, dot = 0.f;
    if (there) {
        const View& x = queries ? p.dout : p.v;
        const T* px = static_cast<const T*>(x.data) + b * x.batch + h * x.head + n * x.point;
        const T* py = queries ? static_cast<const T*>(p.out.data) + b * p.out.batch + h * p.out.head + n * p.out.point : px;
        const T* pr = queries && p.rest.data != nullptr ? static_cast<const T*>(p.rest.data) + b * p.rest.batch + h * p.rest.head + n * p.rest.point : nullptr;
        for (int c = part * 8; c < p.C; c += 32) {
            const Pack<T, 8> a = *reinterpret_cast<const Pack<T, 8>*>(px + c), o = *reinterpret_cast<const Pack<T, 8>*>(py + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float f = to_float(a.v[i]);
                dot = fmaf(f, to_float(o.v[i]), dot);
                if (SCALED) square = fmaf(f, f, square);
            }
            if (pr != nullptr) {
                const Pack<T, 8> r = *reinterpret_cast<const Pack<T, 8>*>(pr + c);
#pragma unroll
                for (int i = 0; i < 8; ++i) dot = fmaf(to_float(a.v[i]), to_float(r.v[i]), dot);
            }
        }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
        if (SCALED) square += __shfl_xor_sync(0xffffffffu, square, o);
    }
    if (queries && part < 2) {
        float lse2 = INFINITY, D = 0.f;
        if (there) {
            const int64_t row = bh * p.Nq + n;
            const float lse = p.lse[row];
            if (lse != -INFINITY) {
                lse2 = lse * LOG2E - SHIFT<T>;
                D = dot;
            }
            if (part == 0) s.lse2[row] = lse2;
            else s.D[row] = D;
        }
        // (1, 1, 1, -lse / scale in parts) against (weight of a key in parts, 1, 1, 1), and (-D in parts) against ones
        const uint2 parts = part == 1 ? extra_parts(-D) : lse2 == INFINITY ? make_uint2(EXTRA_OUT, 0) : extra_parts(-lse2 / p.scale_log2);
        s.extra[(block * 2 + part) * STATS_BLOCK + place] =
            part == 1 ? make_uint4(parts.x, parts.y, 0, 0) : make_uint4(EXTRA_ONES_0, EXTRA_ONES_1 | (parts.x << 16), (parts.x >> 16) | (parts.y << 16), 0);
    }
    if (SCALED) {
        if (threadIdx.x == 0) most = 0;
        __syncthreads();
        // (rows of infinities or NaN, whose own gradients are no numbers, do not count: the others are to be scaled as without them)
        if (there && part == 0 && square < INFINITY) atomicMax(&most, __float_as_uint(sqrtf(square)));
        __syncthreads();
        if (threadIdx.x == 0 && most != 0) atomicMax(s.norms + (b * p.Hk + (queries ? h / p.G : h)) * 2 + (queries ? 0 : 1), most);
    }
}

// ---- backward: dq -------------------------------------------------------------------------------------------------------------

template <int CP> constexpr int dq_smem() { return 2 * 64 * CP * 2 + 4 * BN * CP * 2; }

// A block owns 64 stacked rows (16 per warp) and walks all keys.
template <typename T, int CP>
__global__ void __launch_bounds__(THREADS) attend_dq_kernel(const __grid_constant__ Problem p, const __grid_constant__ Stats st, int tiles) {
    constexpr int BM = 64, NT = BN / 8, CN = CP / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(16) float bias[4][BN];
    const uint32_t tq = s32(smem), ty = tq + BM * CP * 2, tkv = ty + BM * CP * 2;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int tile = blockIdx.x % tiles, bh = blockIdx.x / tiles, b = bh / p.Hk, hk = bh - b * p.Hk;
    const int rows = p.G * p.Nq, row0 = tile * BM;
    const T* kh = static_cast<const T*>(p.k.data) + b * p.k.batch + hk * p.k.head;
    const T* vh = static_cast<const T*>(p.v.data) + b * p.v.batch + hk * p.v.head;
    const float* weights = p.log_weights == nullptr ? nullptr : p.log_weights + b * p.log_weights_batch;
    const int last = (p.Nk + BN - 1) / BN;
    // a weight is read one step before it is stored, so that no step waits for it
    float weight = -INFINITY;
    auto fetch_bias = [&](int j) {
        if (tid < BN) {
            const int n = j * BN + tid;
            weight = j < last && n < p.Nk ? weight2(weights, n) : -INFINITY;
        }
    };
    bool present = false;       // whether any point of this thread's takes part
    auto store_bias = [&](int j) {
        if (tid >= BN) return;
        bias[j & 3][tid] = weight;
        present |= weight != -INFINITY;
    };
    auto load_block = [&](int j) {
        if (j < last) {
            auto take = [&](int r) { return bias[j & 3][r] != -INFINITY; };
            const uint32_t stage = tkv + (j & 1) * 2 * BN * CP * 2;
            load_rows<CP, BN>(stage, kh, p.k.point, j * BN, p.C, take);
            load_rows<CP, BN>(stage + BN * CP * 2, vh, p.v.point, j * BN, p.C, take);
        }
        commit();
    };
    load_stacked<CP>(tq, static_cast<const T*>(p.q.data) + b * p.q.batch + (int64_t)hk * p.G * p.q.head, p.q.head, p.q.point, row0, rows, p.Nq, BM, p.C);
    load_stacked<CP>(ty, static_cast<const T*>(p.dout.data) + b * p.dout.batch + (int64_t)hk * p.G * p.dout.head, p.dout.head, p.dout.point, row0, rows, p.Nq, BM, p.C);
    fetch_bias(0);
    store_bias(0);
    fetch_bias(1);
    store_bias(1);
    fetch_bias(2);
    __syncthreads();
    load_block(0);

    const int64_t first_row = ((int64_t)b * p.Hq + hk * p.G) * p.Nq;        // (stacked rows lie one after the other in the statistics)
    float lse2[2], D[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = row0 + warp * 16 + (lane >> 2) + 8 * r;
        lse2[r] = row < rows ? st.lse2[first_row + row] : INFINITY;
        D[r] = row < rows ? st.D[first_row + row] : 0.f;
    }
    const float factor = ds_scale<T>(st, bh);
    float dq[CN][4];
#pragma unroll
    for (int n = 0; n < CN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) dq[n][i] = 0.f;

    for (int j = 0; j < last; ++j) {
        store_bias(j + 2);
        fetch_bias(j + 3);
        load_block(j + 1);
        wait_group<1>();
        __syncthreads();
        const uint32_t tk = tkv + (j & 1) * 2 * BN * CP * 2, tv = tk + BN * CP * 2;
        float s[NT][4], t[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) { s[n][i] = 0.f; t[n][i] = 0.f; }
#pragma unroll
        for (int ks = 0; ks < CP / 16; ++ks) {
            uint32_t a[4], y[4];
            load_a<CP>(a, tq, warp * 16, ks, lane);
            load_a<CP>(y, ty, warp * 16, ks, lane);
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                uint32_t kb[4], vb[4];
                load_b<CP>(kb, tk, n * 8, ks, lane);
                mma<T>(s[n], a, kb[0], kb[1]);
                mma<T>(s[n + 1], a, kb[2], kb[3]);
                load_b<CP>(vb, tv, n * 8, ks, lane);
                mma<T>(t[n], y, vb[0], vb[1]);
                mma<T>(t[n + 1], y, vb[2], vb[3]);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float2 w = *reinterpret_cast<const float2*>(&bias[j & 3][n * 8 + (lane & 3) * 2]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float pr = ex2(fmaf(s[n][i], p.scale_log2, (i & 1) ? w.y : w.x) - lse2[i >> 1]);
                s[n][i] = pr * ((t[n][i] - D[i >> 1]) * factor);
            }
        }
#pragma unroll
        for (int ks = 0; ks < BN / 16; ++ks) {
            uint32_t a[4], a_lo[4];
            operands<T>(s[2 * ks], s[2 * ks + 1], a, a_lo);
#pragma unroll
            for (int n = 0; n < CN; n += 2) {
                uint32_t kb[4];
                load_bt<CP>(kb, tk, ks * 16, n / 2, lane);
                mma<T>(dq[n], a_lo, kb[0], kb[1]);
                mma<T>(dq[n + 1], a_lo, kb[2], kb[3]);
                mma<T>(dq[n], a, kb[0], kb[1]);
                mma<T>(dq[n + 1], a, kb[2], kb[3]);
            }
        }
        __syncthreads();
    }
    wait_group<0>();
    // (where nothing takes part there is no gradient, not even of a query or for a gradient of infinities or NaN)
    const bool nothing = weights != nullptr && __syncthreads_or(present) == 0;
    const float back = p.scale * ex2(-SHIFT<T>) / factor;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = row0 + warp * 16 + (lane >> 2) + 8 * r;
        if (row >= rows) continue;
        const int g = row / p.Nq;
        T* out = static_cast<T*>(p.dq.data) + b * p.dq.batch + (int64_t)(hk * p.G + g) * p.dq.head + (int64_t)(row - g * p.Nq) * p.dq.point;
#pragma unroll
        for (int n = 0; n < CN; ++n) {
            const int c = n * 8 + (lane & 3) * 2;
            if (c < p.C) *reinterpret_cast<uint32_t*>(out + c) = nothing ? 0u : pack<T>(dq[n][2 * r] * back, dq[n][2 * r + 1] * back);
        }
    }
}

// ---- backward: dk, dv -----------------------------------------------------------------------------------------------------------

// Streamed queries per block: 64, or 32 for wide heads, whose two sums take 128 registers
template <int CP> constexpr int DKDV_QUERIES = CP > 64 ? 32 : 64;
template <int CP> constexpr int dkdv_smem() { return 2 * 64 * CP * 2 + 4 * DKDV_QUERIES<CP> * CP * 2; }

// A block owns 64 keys (16 per warp) and walks the stacked queries of its group.
template <typename T, int CP>
__global__ void __launch_bounds__(THREADS) attend_dkdv_kernel(const __grid_constant__ Problem p, const __grid_constant__ Stats st, int tiles) {
    constexpr int BM = 64, QB = DKDV_QUERIES<CP>, NT = QB / 8, CN = CP / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(16) float2 stats[2][QB];         // lse2, D
    const uint32_t tk = s32(smem), tv = tk + BM * CP * 2, tqy = tv + BM * CP * 2;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int tile = blockIdx.x % tiles, bh = blockIdx.x / tiles, b = bh / p.Hk, hk = bh - b * p.Hk;
    const int rows = p.G * p.Nq, key0 = tile * BM;
    const T* qg = static_cast<const T*>(p.q.data) + b * p.q.batch + (int64_t)hk * p.G * p.q.head;
    const T* yg = static_cast<const T*>(p.dout.data) + b * p.dout.batch + (int64_t)hk * p.G * p.dout.head;
    const float* weights = p.log_weights == nullptr ? nullptr : p.log_weights + b * p.log_weights_batch;
    const int64_t first_row = ((int64_t)b * p.Hq + hk * p.G) * p.Nq;
    const int last = (rows + QB - 1) / QB;
    auto load_block = [&](int j) {
        if (j < last) {
            const uint32_t stage = tqy + (j & 1) * 2 * QB * CP * 2;
            load_stacked<CP>(stage, qg, p.q.head, p.q.point, j * QB, rows, p.Nq, QB, p.C);
            load_stacked<CP>(stage + QB * CP * 2, yg, p.dout.head, p.dout.point, j * QB, rows, p.Nq, QB, p.C);
            if (tid < QB) {
                const int row = j * QB + tid;
                stats[j & 1][tid] = row < rows ? make_float2(st.lse2[first_row + row], st.D[first_row + row]) : make_float2(INFINITY, 0.f);
            }
        }
        commit();
    };
    auto take = [&](int r) { return key0 + r < p.Nk && weight2(weights, key0 + r) != -INFINITY; };
    load_rows<CP, BM>(tk, static_cast<const T*>(p.k.data) + b * p.k.batch + hk * p.k.head, p.k.point, key0, p.C, take);
    load_rows<CP, BM>(tv, static_cast<const T*>(p.v.data) + b * p.v.batch + hk * p.v.head, p.v.point, key0, p.C, take);
    load_block(0);
    float w2[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int n = key0 + warp * 16 + (lane >> 2) + 8 * r;
        w2[r] = n < p.Nk ? weight2(weights, n) : -INFINITY;
    }
    const float factor = ds_scale<T>(st, bh);
    float dk[CN][4], dv[CN][4];
#pragma unroll
    for (int n = 0; n < CN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) { dk[n][i] = 0.f; dv[n][i] = 0.f; }

    for (int j = 0; j < last; ++j) {
        load_block(j + 1);
        wait_group<1>();
        __syncthreads();
        const uint32_t tq = tqy + (j & 1) * 2 * QB * CP * 2, ty = tq + QB * CP * 2;
        float s[NT][4], t[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) { s[n][i] = 0.f; t[n][i] = 0.f; }
#pragma unroll
        for (int ks = 0; ks < CP / 16; ++ks) {
            uint32_t a[4], y[4];
            load_a<CP>(a, tk, warp * 16, ks, lane);
            load_a<CP>(y, tv, warp * 16, ks, lane);
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                uint32_t qb[4], yb[4];
                load_b<CP>(qb, tq, n * 8, ks, lane);
                mma<T>(s[n], a, qb[0], qb[1]);
                mma<T>(s[n + 1], a, qb[2], qb[3]);
                load_b<CP>(yb, ty, n * 8, ks, lane);
                mma<T>(t[n], y, yb[0], yb[1]);
                mma<T>(t[n + 1], y, yb[2], yb[3]);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float4 w = *reinterpret_cast<const float4*>(&stats[j & 1][n * 8 + (lane & 3) * 2]);       // lse2, D of two queries
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][i] = ex2(fmaf(s[n][i], p.scale_log2, w2[i >> 1]) - ((i & 1) ? w.z : w.x));
                t[n][i] = s[n][i] * ((t[n][i] - ((i & 1) ? w.w : w.y)) * factor);
            }
        }
#pragma unroll
        for (int ks = 0; ks < QB / 16; ++ks) {
            uint32_t a[4], a_lo[4];
            operands<T>(s[2 * ks], s[2 * ks + 1], a, a_lo);
            uint32_t d[4], d_lo[4];
            operands<T>(t[2 * ks], t[2 * ks + 1], d, d_lo);
#pragma unroll
            for (int n = 0; n < CN; n += 2) {
                uint32_t yb[4], qb[4];
                load_bt<CP>(yb, ty, ks * 16, n / 2, lane);
                mma<T>(dv[n], a_lo, yb[0], yb[1]);
                mma<T>(dv[n + 1], a_lo, yb[2], yb[3]);
                mma<T>(dv[n], a, yb[0], yb[1]);
                mma<T>(dv[n + 1], a, yb[2], yb[3]);
                load_bt<CP>(qb, tq, ks * 16, n / 2, lane);
                mma<T>(dk[n], d_lo, qb[0], qb[1]);
                mma<T>(dk[n + 1], d_lo, qb[2], qb[3]);
                mma<T>(dk[n], d, qb[0], qb[1]);
                mma<T>(dk[n + 1], d, qb[2], qb[3]);
            }
        }
        __syncthreads();
    }
    wait_group<0>();
    const float unshift = ex2(-SHIFT<T>), back = p.scale * unshift / factor;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int n_key = key0 + warp * 16 + (lane >> 2) + 8 * r;
        if (n_key >= p.Nk) continue;
        const bool left_out = w2[r] == -INFINITY;       // (its sums are NaN if a query or a gradient is infinite or NaN)
        T* k_out = static_cast<T*>(p.dk.data) + b * p.dk.batch + hk * p.dk.head + (int64_t)n_key * p.dk.point;
        T* v_out = static_cast<T*>(p.dv.data) + b * p.dv.batch + hk * p.dv.head + (int64_t)n_key * p.dv.point;
#pragma unroll
        for (int n = 0; n < CN; ++n) {
            const int c = n * 8 + (lane & 3) * 2;
            if (c >= p.C) continue;
            *reinterpret_cast<uint32_t*>(k_out + c) = left_out ? 0u : pack<T>(dk[n][2 * r] * back, dk[n][2 * r + 1] * back);
            *reinterpret_cast<uint32_t*>(v_out + c) = left_out ? 0u : pack<T>(dv[n][2 * r] * unshift, dv[n][2 * r + 1] * unshift);
        }
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------------------

template <typename K>
cudaError_t allow(K kernel, int bytes) {       // (48 KB hold the static arrays too)
    return bytes > 40 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) : cudaSuccess;
}
bool few_rows(const Problem& p) { return p.G * (int64_t)p.Nq <= 16; }
int forward_tiles(const Problem& p) { return (int)(((int64_t)p.G * p.Nq + (few_rows(p) ? 15 : 63)) / (few_rows(p) ? 16 : 64)); }

template <typename T, int CP, int WM>
cudaError_t forward_as(const Problem& p, int splits, float* partials, cudaStream_t stream) {
    const int tiles = forward_tiles(p);
    cudaError_t e = allow(attend_forward_kernel<T, CP, WM>, forward_smem<CP, WM>());
    if (e != cudaSuccess) return e;
    attend_forward_kernel<T, CP, WM><<<(unsigned)((int64_t)p.B * p.Hk * tiles * splits), THREADS, forward_smem<CP, WM>(), stream>>>(p, tiles, splits, splits > 1 ? partials : nullptr);
    return cudaGetLastError();
}
template <typename T, int CP>
cudaError_t dq_as(const Problem& p, const Stats& s, cudaStream_t stream) {
    const int tiles = (int)(((int64_t)p.G * p.Nq + 63) / 64);
    cudaError_t e = allow(attend_dq_kernel<T, CP>, dq_smem<CP>());
    if (e != cudaSuccess) return e;
    attend_dq_kernel<T, CP><<<(unsigned)((int64_t)p.B * p.Hk * tiles), THREADS, dq_smem<CP>(), stream>>>(p, s, tiles);
    return cudaGetLastError();
}
template <typename T, int CP>
cudaError_t dkdv_as(const Problem& p, const Stats& s, cudaStream_t stream) {
    const int tiles = (p.Nk + 63) / 64;
    cudaError_t e = allow(attend_dkdv_kernel<T, CP>, dkdv_smem<CP>());
    if (e != cudaSuccess) return e;
    attend_dkdv_kernel<T, CP><<<(unsigned)((int64_t)p.B * p.Hk * tiles), THREADS, dkdv_smem<CP>(), stream>>>(p, s, tiles);
    return cudaGetLastError();
}
template <typename F>
cudaError_t by_width(int C, F f) {
    return C <= 32 ? f(std::integral_constant<int, 32>()) : C <= 64 ? f(std::integral_constant<int, 64>()) : f(std::integral_constant<int, 128>());
}

}  // namespace

// Blocks that share the keys of a tile: until the GPU has four blocks per SM, with at least four blocks of 64 keys each.
int forward_splits(const Problem& p, int sms) {
    const int64_t tiles = (int64_t)p.B * p.Hk * forward_tiles(p);
    const int64_t blocks = (p.Nk + BN - 1) / BN;
    if (tiles == 0 || blocks == 0 || tiles >= 2 * sms) return 1;
    return (int)std::max<int64_t>(1, std::min(blocks / 4, 4 * sms / tiles));
}

cudaError_t launch_join(const Problem& p, sna_dtype_t dtype, int splits, const float* partials, cudaStream_t stream) {
    const int64_t rows = rows_of(p);
    const bool block_per_row = rows <= 1024;
    const unsigned blocks = (unsigned)(block_per_row ? rows : (rows + JOIN_WARPS - 1) / JOIN_WARPS);
    auto run = [&](auto t) {
        using T = decltype(t);
        return launch_dependent(block_per_row ? attend_join_kernel<T, true> : attend_join_kernel<T, false>, blocks, 32 * JOIN_WARPS, 0, stream, p, splits, partials);
    };
    return dtype == SNA_BFLOAT16 ? run(__nv_bfloat16()) : run(__half());
}

cudaError_t launch_forward(const Problem& p, sna_dtype_t dtype, int splits, float* partials, cudaStream_t stream) {
    return by_width(p.C, [&](auto width) {
        constexpr int CP = decltype(width)::value;
        if (dtype == SNA_BFLOAT16) return few_rows(p) ? forward_as<__nv_bfloat16, CP, 1>(p, splits, partials, stream) : forward_as<__nv_bfloat16, CP, 4>(p, splits, partials, stream);
        return few_rows(p) ? forward_as<__half, CP, 1>(p, splits, partials, stream) : forward_as<__half, CP, 4>(p, splits, partials, stream);
    });
}

cudaError_t launch_selection(const Problem& p, const Selection& sel, cudaStream_t stream) {
    attend_select_kernel<<<(unsigned)select_blocks_of(p), SELECT_POINTS, 0, stream>>>(p, sel);
    return cudaGetLastError();
}

cudaError_t launch_statistics(const Problem& p, const Stats& s, const Selection& sel, sna_dtype_t dtype, cudaStream_t stream) {
    const int64_t query_blocks = query_blocks_of(p), key_blocks = (int64_t)p.B * p.Hk * ((p.Nk + STATS_BLOCK - 1) / STATS_BLOCK);
    const int64_t weight_blocks = sel.taken != nullptr ? select_blocks_of(p) : weight_blocks_of(p, false), blocks = weight_blocks + query_blocks + (dtype == SNA_FLOAT16 ? key_blocks : 0);
    if (blocks == 0) return cudaSuccess;
    if (dtype == SNA_BFLOAT16) {
        attend_statistics_kernel<__nv_bfloat16><<<(unsigned)blocks, 256, 0, stream>>>(p, s, sel, query_blocks, weight_blocks);
    } else {
        const cudaError_t e = cudaMemsetAsync(s.norms, 0, (size_t)p.B * p.Hk * 2 * sizeof(uint32_t), stream);
        if (e != cudaSuccess) return e;
        attend_statistics_kernel<__half><<<(unsigned)blocks, 256, 0, stream>>>(p, s, sel, query_blocks, weight_blocks);
    }
    return cudaGetLastError();
}

cudaError_t launch_backward_dq(const Problem& p, const Stats& s, sna_dtype_t dtype, cudaStream_t stream) {
    return by_width(p.C, [&](auto width) {
        constexpr int CP = decltype(width)::value;
        return dtype == SNA_BFLOAT16 ? dq_as<__nv_bfloat16, CP>(p, s, stream) : dq_as<__half, CP>(p, s, stream);
    });
}

cudaError_t launch_backward_dkdv(const Problem& p, const Stats& s, sna_dtype_t dtype, cudaStream_t stream) {
    return by_width(p.C, [&](auto width) {
        constexpr int CP = decltype(width)::value;
        return dtype == SNA_BFLOAT16 ? dkdv_as<__nv_bfloat16, CP>(p, s, stream) : dkdv_as<__half, CP>(p, s, stream);
    });
}

}  // namespace attend
}  // namespace sna
