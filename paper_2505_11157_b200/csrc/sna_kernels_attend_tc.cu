// The 16-bit attention's kernels for many rows, on tcgen05 / TMEM / TMA (formulas: sna_kernels_attend.cu).
//
// Specialised warps run side by side, coupled by mbarriers only.  A thread of the element-wise warps owns a whole row of a tile, so that
// maxima and sums of a row need no exchange; operands of the second products go back to TMEM as 16-bit pairs.
//
// Every accumulator has one issuing thread and all sums are taken in a fixed order: results are reproducible bit for bit.  Every wait is
// bounded; one that runs out sets the device's status word (sna_layer_check), and the block leaves after another bounded wait for the copies
// and MMAs that it has under way.
#include <algorithm>
#include <type_traits>

#include "sna_attend_tc.cuh"

namespace sna {
namespace attend {
namespace {

__device__ int g_status;        // non-zero: a bounded wait has run out since the last check

// A thread block's tile and its piece of the streamed side.
struct Piece {
    int tile, bh, part, parts;
    int64_t local;          // of a tile in pieces: its number among them
    __device__ __forceinline__ Piece(const Split& cut, int tiles, int64_t block) {
        const int64_t over = block - cut.full;
        parts = over < 0 ? 1 : cut.parts;
        local = over < 0 ? 0 : over / parts;
        part = over < 0 ? 0 : (int)(over - local * parts);
        const int64_t index = over < 0 ? block : cut.full + local;
        bh = (int)(index / tiles);
        tile = (int)(index - (int64_t)bh * tiles);
    }
};

constexpr int TILE = 128;       // rows of a tile, points of a block
constexpr int SLAB = TILE * 128;        // bytes of 128 points x 64 channels

__device__ __forceinline__ bool all_lanes(bool ok) { return __all_sync(0xffffffffu, ok); }
// One arrival per warp, for what its lanes have read from or written to TMEM.  (32 arrivals on one barrier are carried out one after the other.)
__device__ __forceinline__ void warp_arrive(uint32_t bar, int lane) {
    tm_before();
    __syncwarp();
    if (lane == 0) mb_arrive(bar);
}

// ---- forward ---------------------------------------------------------------------------------------------------------------
//
// A block owns two tiles of 128 queries of one head and walks the keys in blocks of 128:
//   warp 8       TMA: q once, then k and v blocks into rings of stages
//   warps 9, 11  MMAs of tile 0 and 1: S = Q K^T of the next block, O += P V of this one, in halves of 64 points as P gets ready
//   warp 10      weights of the next block's points; zeroes k and v rows of points left out
//   warps 0-3 and 4-7  softmax of tile 0 and 1, thread = row: S from TMEM, P back.  The row's reference moves (and O is scaled in TMEM)
//                only when its maximum has grown by 2^8: then the sums are still far from overflow, and most blocks skip the correction.
// Narrow heads leave TMEM columns for P beside S: S of the next block is then computed during this block's softmax.  Wide ones keep P
// in S's columns; while one tile's products run, the other tile's softmax does.
// What bounds them: latencies.  Eight softmax warps keep the special-function unit 52 %, the tensor pipe 34 % and the issue slots 50 % busy (heads of 64); with heads of
// 128 it is the chain of a tile's softmax and products, 3200 cycles per block and pair of tiles, of which the tensor pipe works 2000.  Tried and not kept (64x128, B = 2,
// four heads of 32, 193 us): the two tiles taking turns with their exponentials 225; four groups with half a row per thread, whose scores do not fit
// their 104 registers, 240; the next block's scores loaded and their maxima found between this block's exponentials 213.
// A point's weight is one more step of the first product: its parts against ones.  (Added per element, with the weights read from shared memory, it
// cost 40 % of the time: 64x128, B = 2, eight heads of 128, 683 us against 486 without weights.)
constexpr int FWD_THREADS = 384;

template <int D> struct Forward {
    static constexpr bool P_APART = D == 64;
    static constexpr int SLABS = D / 64, STAGES = D == 64 ? 4 : 2, TILE_BYTES = SLABS * SLAB, EXTRA_BYTES = TILE * 32;
    static constexpr int OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + STAGES * TILE_BYTES, OFF_ONES = OFF_V + STAGES * TILE_BYTES, OFF_W = OFF_ONES + EXTRA_BYTES;
    static constexpr size_t SMEM = OFF_W + STAGES * EXTRA_BYTES + 1024;
    // TMEM columns
    static constexpr int T_P = P_APART ? 256 : 0, P_STEP = P_APART ? 64 : 128, T_O = P_APART ? 384 : 256;
    enum { Q_FULL = 0, K_FULL = 2, V_FULL = K_FULL + STAGES, K_FREE = V_FULL + STAGES, V_FREE = K_FREE + STAGES, K_READY = V_FREE + STAGES,
           V_READY = K_READY + STAGES, S_FULL = V_READY + STAGES, S_FREE = S_FULL + 2, P_READY = S_FREE + 2 /* [tile][half] */, O_DONE = P_READY + 4, DRAIN = O_DONE + 2, COUNT = DRAIN + 2 };
};

// Eight values rounded to 16 bits, and what rounding took from them.
template <typename T>
__device__ __forceinline__ void store8(T* out, T* rest, const float (&y)[8]) {
    uint32_t x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = pack16<T>(y[2 * k], y[2 * k + 1]);
    *reinterpret_cast<uint4*>(out) = make_uint4(x[0], x[1], x[2], x[3]);
    if (rest == nullptr) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float a, b;
        unpack2(pair_of<T>(x[k]), a, b);
        x[k] = pack16<T>(y[2 * k] - a, y[2 * k + 1] - b);
    }
    *reinterpret_cast<uint4*>(rest) = make_uint4(x[0], x[1], x[2], x[3]);
}

// Two values rounded to 16 bits, and if FINE what rounding takes from them.
template <typename T, bool FINE>
__device__ __forceinline__ uint32_t pack_parts(float x, float y, uint32_t& rest) {
    const uint32_t word = pack16<T>(x, y);
    if (FINE) {
        float a, b;
        unpack2(pair_of<T>(word), a, b);
        rest = pack16<T>(x - a, y - b);
    }
    return word;
}

// Rounded to float16, weights up to 2^8 times the reference's must stay finite: 2^(8 + 7) < 65504.
template <typename T> constexpr float FORWARD_SHIFT = 0.f;
template <> constexpr float FORWARD_SHIFT<__half> = 7.f;
constexpr float GROWTH = 8.f;
constexpr int BY_FMA = 4;               // one pair of this many takes its exponentials on the FMA pipe (us in the case above: none 204, 1 in 3 196, 1 in 4 194, 1 in 2 213)
constexpr float NOTHING = -1e31f;       // scores below belong to points left out

template <typename T, int D, bool WEIGHTS>
__global__ void __launch_bounds__(FWD_THREADS, 1)
attend_forward_tc_kernel(const __grid_constant__ Problem p, const __grid_constant__ Selection sel, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                         const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_k_sel, const __grid_constant__ CUtensorMap map_v_sel, int tiles,
                         const __grid_constant__ Split cut, float* partials) {
    using F = Forward<D>;
    allow_dependents();
    extern __shared__ unsigned char raw[];
    unsigned char* base = (unsigned char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    __shared__ unsigned long long bars[F::COUNT];
    __shared__ uint32_t tmem_s;
    __shared__ int fail_s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Piece piece(cut, tiles, blockIdx.x);
    const int part = piece.part, parts = piece.parts, tile = piece.tile, bh = piece.bh;
    const int b = bh / p.Hq, h = bh - b * p.Hq, hk = h / p.G;
    const int row0 = tile * 2 * TILE, halves = row0 + TILE < p.Nq ? 2 : 1;
    const int steps = (p.C + 15) / 16, slabs = (p.C + 63) / 64;
    auto bar = [&](int i) { return s32(&bars[i]); };

    if (tid == 0) {
        for (int i = 0; i < F::COUNT; ++i)
            mb_init(bar(i), i >= F::S_FREE && i < F::O_DONE ? 4 : i >= F::K_FREE && i < F::K_READY ? halves : 1);
        fail_s = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s32(&tmem_s)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (WEIGHTS) {
        // the ones, and zeros behind the weights' parts
        for (int e = tid; e < F::EXTRA_BYTES / 16; e += FWD_THREADS)
            *reinterpret_cast<uint4*>(base + F::OFF_ONES + e * 16) = (e & 8) ? make_uint4(0, 0, 0, 0) : make_uint4(EXTRA_ONES_0, EXTRA_ONES_1, 0, 0);
        for (int e = tid; e < F::STAGES * F::EXTRA_BYTES / 16; e += FWD_THREADS) *reinterpret_cast<uint4*>(base + F::OFF_W + e * 16) = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    tm_before();
    __syncthreads();
    tm_after();
    const uint32_t tm = tmem_s;
    bool ok = true;

    int Nk = p.Nk;
    if (WEIGHTS) {
        wait_for_previous();
        if (sel.taken != nullptr) Nk = sel.taken[b];
    }
    const bool apart = WEIGHTS && Nk != p.Nk;
    const int blocks = (Nk + TILE - 1) / TILE;
    const int first = (int)((int64_t)blocks * part / parts), count = (int)((int64_t)blocks * (part + 1) / parts) - first;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 8 && elect_one()) {
            // ---------------------------------------------------------------- TMA
            for (int t = 0; t < halves; ++t) {
                mb_expect(bar(F::Q_FULL + t), slabs * SLAB);
                for (int s = 0; s < slabs; ++s) tma_load(s32(base) + t * F::TILE_BYTES + s * SLAB, &map_q, s * 64, row0 + t * TILE, h, b, bar(F::Q_FULL + t));
            }
            int it = 0;
            const CUtensorMap *keys = apart ? &map_k_sel : &map_k, *values = apart ? &map_v_sel : &map_v;
            for (; it < count && ok; ++it) {
                const int st = it % F::STAGES, turn = it / F::STAGES;
                if (turn > 0) ok = mb_wait(bar(F::K_FREE + st), (turn - 1) & 1, ok);
                if (!ok) break;
                mb_expect(bar(F::K_FULL + st), slabs * SLAB);
                for (int s = 0; s < slabs; ++s) tma_load(s32(base) + F::OFF_K + st * F::TILE_BYTES + s * SLAB, keys, s * 64, (first + it) * TILE, hk, b, bar(F::K_FULL + st));
                if (turn > 0) ok = mb_wait(bar(F::V_FREE + st), (turn - 1) & 1, ok);
                if (!ok) break;
                mb_expect(bar(F::V_FULL + st), slabs * SLAB);
                for (int s = 0; s < slabs; ++s) tma_load(s32(base) + F::OFF_V + st * F::TILE_BYTES + s * SLAB, values, s * 64, (first + it) * TILE, hk, b, bar(F::V_FULL + st));
            }
            // the copies under way (all there already if all went well)
            for (int t = 0; t < halves; ++t) mb_wait(bar(F::Q_FULL + t), 0, true);
            for (int back = 0; back <= F::STAGES && back <= it; ++back) {
                const int i = it - back, st = i % F::STAGES, turn = i / F::STAGES;
                if (i >= count) continue;
                mb_wait(bar(F::K_FULL + st), turn & 1, i < it || !ok);
                if (i < it) mb_wait(bar(F::V_FULL + st), turn & 1, true);
            }
        } else if ((warp == 9 || (F::P_APART && warp == 11 && halves == 2)) && elect_one()) {
            // ---------------------------------------------------------------- MMAs
            const uint32_t ids = idesc<T>(TILE, false), idw = idesc<__nv_bfloat16>(TILE, false), ido = idesc<T>(steps * 16, true);
            const uint32_t dq = desc_channels(s32(base)), dk = desc_channels(s32(base) + F::OFF_K), dv = desc_points(s32(base) + F::OFF_V, SLAB);
            const uint32_t dones = desc_extra(s32(base) + F::OFF_ONES), dw = desc_extra(s32(base) + F::OFF_W);
            auto scores = [&](int t, int it) {
                const int st = it % F::STAGES;
                if (!mb_wait(bar((WEIGHTS ? F::K_READY : F::K_FULL) + st), (it / F::STAGES) & 1, true)) return false;
                const uint32_t to = tm + t * TILE, a = dq + t * (F::TILE_BYTES >> 4), k = dk + st * (F::TILE_BYTES >> 4);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    if (ks < steps) mma_ss(to, a + (ks >> 2) * (SLAB >> 4) + (ks & 3) * 2, k + (ks >> 2) * (SLAB >> 4) + (ks & 3) * 2, ids, ks > 0);
                if (WEIGHTS) mma_ss<DESC_EXTRA_HIGH>(to, dones, dw + st * (F::EXTRA_BYTES >> 4), idw, 1);
                mma_commit(bar(F::S_FULL + t));
                mma_commit(bar(F::K_FREE + st));
                return true;
            };
            auto values = [&](int t, int it) {
                const int st = it % F::STAGES;
                if (!mb_wait(bar((WEIGHTS ? F::V_READY : F::V_FULL) + st), (it / F::STAGES) & 1, true)) return false;
                const uint32_t to = tm + F::T_O + t * D, a = tm + F::T_P + t * F::P_STEP, v = dv + st * (F::TILE_BYTES >> 4);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (!mb_wait(bar(F::P_READY + 2 * t + half), it & 1, true)) return false;
                    tm_after();
#pragma unroll
                    for (int kk = 4 * half; kk < 4 * half + 4; ++kk) mma_ts(to, a + kk * 8, v + kk * (2048 >> 4), ido, it > 0 || kk > 0);
                }
                mma_commit(bar(F::O_DONE + t));
                mma_commit(bar(F::V_FREE + st));
                return true;
            };
            if constexpr (F::P_APART) {
                const int t = warp == 9 ? 0 : 1;
                ok = mb_wait(bar(F::Q_FULL + t), 0, true) && (count == 0 || scores(t, 0));
                for (int it = 0; it < count && ok; ++it) {
                    if (it + 1 < count) {
                        ok = mb_wait(bar(F::S_FREE + t), it & 1, true);
                        if (!ok) break;
                        tm_after();
                        ok = scores(t, it + 1);
                    }
                    ok = ok && values(t, it);
                }
            } else {
                // (one thread for both tiles: with one each, the two softmaxes drift into step and wait together; 64x128, B = 2, eight heads of 128: 708 us)
                for (int t = 0; t < halves && ok; ++t) ok = mb_wait(bar(F::Q_FULL + t), 0, true) && (count == 0 || scores(t, 0));
                for (int it = 0; it < count && ok; ++it)
                    for (int t = 0; t < halves && ok; ++t) ok = values(t, it) && (it + 1 >= count || scores(t, it + 1));
            }
            mma_commit(bar(F::DRAIN + (warp == 9 ? 0 : 1)));
            mb_wait(bar(F::DRAIN + (warp == 9 ? 0 : 1)), 0, true);
        } else if (WEIGHTS && warp == 10) {
            // ---------------------------------------------------------------- weights
            const float* weights = apart ? sel.weights + (int64_t)b * p.Nk : p.log_weights + b * p.log_weights_batch;
            const float unscale = 1.f / p.scale;
            float w[4];
            auto fetch = [&](int it) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = (first + it) * TILE + i * 32 + lane;
                    w[i] = n >= Nk ? -INFINITY : weights[n];
                }
            };
            if (count > 0) fetch(0);
            for (int it = 0; it < count && ok; ++it) {
                const int st = it % F::STAGES;
                const uint32_t phase = (it / F::STAGES) & 1;
                uint32_t gone[4], any = 0;
                uint2 parts[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool out = w[i] <= EXCLUDED;
                    gone[i] = __ballot_sync(0xffffffffu, out && (first + it) * TILE + i * 32 + lane < Nk);
                    any |= gone[i];
                    parts[i] = out ? make_uint2(EXTRA_OUT, 0) : extra_parts(w[i] * unscale);
                }
                if (it + 1 < count) fetch(it + 1);
                ok = all_lanes(mb_wait(bar(F::K_FULL + st), phase, ok));        // (the stage's last scores are done, too)
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<uint2*>(base + F::OFF_W + st * F::EXTRA_BYTES + extra_at(i * 32 + lane)) = parts[i];
                if (any)
#pragma unroll
                    for (int i = 0; i < 4; ++i) zero_rows(base + F::OFF_K + st * F::TILE_BYTES, slabs, SLAB, i, gone[i], lane);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mb_arrive(bar(F::K_READY + st));
                ok = all_lanes(mb_wait(bar(F::V_FULL + st), phase, ok));
                if (!ok) break;
                if (any)
#pragma unroll
                    for (int i = 0; i < 4; ++i) zero_rows(base + F::OFF_V + st * F::TILE_BYTES, slabs, SLAB, i, gone[i], lane);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mb_arrive(bar(F::V_READY + st));
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int t = warp >> 2;
        if (t < halves) {
            // ------------------------------------------------------------ softmax
            const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
            const uint32_t ts = tm + t * TILE + lanes, tp = tm + F::T_P + t * F::P_STEP + lanes, to = tm + F::T_O + t * D + lanes;
            const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2);
            float ref = -INFINITY, l = 0.f;
            for (int it = 0; it < count && ok; ++it) {
                uint32_t s[TILE];
                ok = all_lanes(mb_wait(bar(F::S_FULL + t), it & 1, ok));
                if (!ok) break;
                tm_after();
#pragma unroll
                for (int c = 0; c < 4; ++c) tm_ld32(s + 32 * c, ts + 32 * c);
                tm_ld_wait();
                if (F::P_APART) {
                    warp_arrive(bar(F::S_FREE + t), lane);
                }
                if (!WEIGHTS && (first + it + 1) * TILE > p.Nk) {
                    const int there = p.Nk - (first + it) * TILE;       // (the scale is positive)
#pragma unroll
                    for (int i = 0; i < TILE; ++i)
                        if (i >= there) s[i] = 0xff800000u;
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < TILE; i += 8)
#pragma unroll
                    for (int k = 0; k < 4; ++k) top[k] = max3(top[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
                float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.scale_log2;
                if (WEIGHTS && now < NOTHING) now = -INFINITY;
                const bool grown = now > ref + GROWTH;       // (also the first finite maximum: the reference is -infinity until then)
                if (__any_sync(0xffffffffu, grown)) {
                    const float factor = grown ? ex2(ref - now) : 1.f;
                    l *= factor;
                    ref = grown ? now : ref;
                    if (it > 0) {
                        ok = all_lanes(mb_wait(bar(F::O_DONE + t), (it - 1) & 1, ok));
                        if (!ok) break;
                        tm_after();
                        const uint64_t factor2 = pack2(factor, factor);
                        for (int c = 0; c < steps * 16; c += 32) {
                            uint32_t o[32];
                            tm_ld32(o, to + c);
                            tm_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                float x, y;
                                unpack2(mul2(pack2(__uint_as_float(o[i]), __uint_as_float(o[i + 1])), factor2), x, y);
                                o[i] = __float_as_uint(x); o[i + 1] = __float_as_uint(y);
                            }
                            tm_st32(to + c, o);
                        }
                    }
                }
                const float off = FORWARD_SHIFT<T> - (ref == -INFINITY ? 0.f : ref);
                const uint64_t off2 = pack2(off, off);
                uint64_t sum2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t pr[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const uint64_t x2 = fma2(pack2(__uint_as_float(s[64 * half + 2 * i]), __uint_as_float(s[64 * half + 2 * i + 1])), scale2, off2);
                        float x, y;
                        if (i % BY_FMA == BY_FMA - 1) {
                            exp2_by_fma(x2, x, y);
                        } else {
                            unpack2(x2, x, y);
                            x = ex2(x); y = ex2(y);
                        }
                        sum2[i & 1] = add2(sum2[i & 1], pack2(x, y));
                        pr[i] = pack16<T>(x, y);
                    }
                    if (F::P_APART && half == 0 && it > 0) {
                        ok = all_lanes(mb_wait(bar(F::O_DONE + t), (it - 1) & 1, ok));      // the last block's P has been read
                        if (!ok) break;
                    }
                    tm_st32(tp + 32 * half, pr);
                    tm_st_wait();
                    warp_arrive(bar(F::P_READY + 2 * t + half), lane);
                }
                float a0, a1, a2, a3;
                unpack2(sum2[0], a0, a1);
                unpack2(sum2[1], a2, a3);
                l += (a0 + a1) + (a2 + a3);
            }
            if (ok && count > 0) ok = all_lanes(mb_wait(bar(F::O_DONE + t), (count - 1) & 1, ok));
            if (ok) {
                tm_after();
                bool nothing = count == 0;
                if (WEIGHTS && !apart && __any_sync(0xffffffffu, l != l)) {
                    // A query of infinities or NaN makes S NaN against the zeros of points left out, too: with those alone its row is one without points.
                    const float* weights = p.log_weights + b * p.log_weights_batch;
                    const int end = min(Nk, (first + count) * TILE);
                    nothing = true;
                    for (int n = first * TILE; n < end && nothing; n += 32)
                        nothing = __all_sync(0xffffffffu, n + lane >= end || weights[n + lane] <= EXCLUDED);
                    if (nothing) { ref = -INFINITY; l = 0.f; }
                }
                const int row = row0 + t * TILE + (warp & 3) * 32 + lane;
                const int64_t at = ((int64_t)b * p.Hq + h) * p.Nq + row;
                const int64_t rest = cut.rest() * 2 * TILE, local = piece.local * 2 * TILE + t * TILE + (warp & 3) * 32 + lane;
                const bool there = row < p.Nq;
                const bool none = ref == -INFINITY && l == l;        // (not a row of NaN)
                const float inverse = none ? 0.f : 1.f / l;
                if (there) {
                    const float lse2 = none ? -INFINITY : ref + log2f(l) - FORWARD_SHIFT<T>;
                    if (parts > 1) partials[parts * rest * p.C + part * rest + local] = lse2;
                    else if (p.lse != nullptr) p.lse[at] = lse2 * LN2;
                }
                for (int c = 0; c < p.C; c += 32) {
                    uint32_t o[32];
                    if (!nothing) {
                        tm_ld32(o, to + c);
                        tm_ld_wait();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0;
                    }
                    if (!there) continue;
                    if (parts > 1) {
                        float* out = partials + (part * rest + local) * p.C + c;
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            if (c + i < p.C)
                                *reinterpret_cast<float4*>(out + i) = make_float4(__uint_as_float(o[i]) * inverse, __uint_as_float(o[i + 1]) * inverse,
                                                                                  __uint_as_float(o[i + 2]) * inverse, __uint_as_float(o[i + 3]) * inverse);
                    } else {
                        T* out = static_cast<T*>(p.out.data) + b * p.out.batch + h * p.out.head + row * p.out.point + c;
                        T* rest_out = p.rest.data == nullptr ? nullptr : static_cast<T*>(p.rest.data) + b * p.rest.batch + h * p.rest.head + row * p.rest.point;
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            if (c + i < p.C) {
                                float y[8];
#pragma unroll
                                for (int k = 0; k < 8; ++k) y[k] = __uint_as_float(o[i + k]) * inverse;
                                store8<T>(out + i, rest_out == nullptr ? nullptr : rest_out + c + i, y);
                            }
                    }
                }
            }
        }
    }
    if (!ok) atomicExch(&fail_s, 1);
    tm_before();
    __syncthreads();
    if (fail_s && tid == 0) atomicExch(&g_status, 1);
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tm), "r"(512));
}

// ---- backward -----------------------------------------------------------------------------------------------------------------
//
// dq and dk, dv are the same walk with the sides exchanged.  A block owns 128 rows x (queries: dq; keys: dk, dv) with their operands A1 (q or k) and
// A2 (dout or v), and walks the other side's points in blocks of 64, B1 (k or q) and B2 (v or dout):
//   S = A1 B1^T, T = A2 B2^T;  p = exp(S - lse), ds = p (T - D);  acc1 += ds B1 (dq or dk);  dk, dv: acc2 += p B2 (dv)
//   warp 16  TMA of the blocks
//   warps 17, 19  MMAs, as soon as block j has left the columns: dv of block j and S of block j + 2 (dq: S alone, when S has been read); dk or dq of
//            block j and T of block j + 2.  (One thread for all of them was busy all the time: a wait costs it 60 cycles or more even if it need not wait.)
//   warp 18  dq: if points are left out, zeroes their rows of the block (their weights come with it)
//   warps 0-15  element-wise: a group of four warps takes one half of the columns of the blocks of even or of odd number, thread = row; p while T is computed;
//            p and ds go back over S and T, each half over its own.  (Two groups, with whole rows per thread, were bound by latencies: issue slots 39 %,
//            special-function unit 55 % busy.)
// Blocks of 64 points need two buffers of S and T to keep both sides busy: 256 of the 512 columns.  An MMA of 64 columns that reads its
// A operand from shared memory is bound by that (6 KB at 128 bytes per clock: 48 cycles instead of 32), so A1 and A2 are kept in TMEM; only for dk, dv of wide
// heads, whose two sums take the other 256 columns, are they in shared memory.
// FINE: p and ds are held in two 16-bit parts, the second in the columns that the 32-bit scores leave free.
constexpr int BWD_THREADS = 640, BLOCK = 64, BSLAB = BLOCK * 128;

template <int D, bool DKDV> struct Backward {
    static constexpr bool A_IN_TMEM = D == 64 || !DKDV;
    static constexpr int SLABS = D / 64, STAGES = D == 64 ? 8 : A_IN_TMEM ? 6 : 4, STAGE_BYTES = 2 * SLABS * BSLAB, A_BYTES = A_IN_TMEM ? 0 : 2 * SLABS * SLAB;
    // Extra steps of the first products (see the forward kernel): one tile of 16 channels for each operand that takes part.
    //   dq      S: ones x weights of the block's points
    //   dk, dv  S: (weight of the row, ones) x (ones, -lse / scale of the block's queries), so that p = exp2(scale_log2 S); T: ones x -D, so that it is t - D
    // (the streamed side's are written by the statistics kernel and copied with the block; with a warp of this kernel that made them, it was that warp's 1180
    // cycles per block that the others waited for)
    static constexpr int EXTRA_A = TILE * 32, EXTRA_B = BLOCK * 16, EXTRAS = DKDV ? 2 : 1;
    static constexpr int OFF_XA = A_BYTES + STAGES * STAGE_BYTES, OFF_XB = OFF_XA + EXTRAS * EXTRA_A;
    static constexpr size_t SMEM = OFF_XB + STAGES * EXTRAS * EXTRA_B + 1024;
    // TMEM columns: buffers of (S, T), sums, operands
    static constexpr int T_BUF = 0, T_ACC = 256, T_A = T_ACC + (DKDV ? 2 : 1) * D;
    static_assert(T_A + (A_IN_TMEM ? D : 0) <= 512, "TMEM");
    enum { A_FULL = 0, A_READY = 1, FULL = 2, READY = FULL + STAGES, FREE = READY + STAGES, S_FULL = FREE + STAGES, T_FULL = S_FULL + 2,
           S_DONE = T_FULL + 2 /* S read (dq) or P ready (dk, dv) */, D_READY = S_DONE + 2, ACC_DONE = D_READY + 2, COUNT };
};

// dq's tiles, or dk's and dv's
struct Side {
    Split cut;
    int tiles;          // of a head
    float* partials;
};
// In boxes of a streamed block: queries and their gradients (for dk, dv), keys and values (for dq).  In boxes of a tile: keys and values, where dk, dv has them in
// shared memory.  The selected ones are there if there is a selection.
struct BackwardMaps {
    CUtensorMap q, dout, k, v, k_sel, v_sel, k_tile, v_tile, k_sel_tile, v_sel_tile;
};

template <typename T, int D, bool DKDV, bool WEIGHTS, bool FINE>
__device__ __forceinline__ void backward_block(const Problem& p, const Stats& stats, const Selection& sel, const BackwardMaps& maps, const Side& side, int64_t block) {
    using K = Backward<D, DKDV>;
    const Split& cut = side.cut;
    float* const partials = side.partials;
    constexpr bool EXTRA = DKDV || WEIGHTS;
    static_assert(BLOCK == STATS_BLOCK, "the statistics kernel's blocks");
    extern __shared__ unsigned char raw[];
    unsigned char* base = (unsigned char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    __shared__ unsigned long long bars[K::COUNT];
    __shared__ uint32_t tmem_s;
    __shared__ int fail_s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Piece piece(cut, side.tiles, block);
    const int tile = piece.tile, bh = piece.bh;
    const int heads = DKDV ? p.Hk : p.Hq, b = bh / heads, head = bh - b * heads, hk = DKDV ? head : head / p.G;
    const int Nk = WEIGHTS && sel.taken != nullptr ? sel.taken[b] : p.Nk;
    const bool apart = WEIGHTS && Nk != p.Nk;
    const int row0 = tile * TILE, N = DKDV ? Nk : p.Nq, M = DKDV ? p.Nq : Nk;       // rows, streamed points
    const int per_head = (M + BLOCK - 1) / BLOCK, total = DKDV ? p.G * per_head : per_head;
    // blocks of the streamed side: `begin` and on, numbered from 0 in the pipeline
    const int begin = (int)((int64_t)total * piece.part / piece.parts), count = (int)((int64_t)total * (piece.part + 1) / piece.parts) - begin;
    const int steps = (p.C + 15) / 16, slabs = (p.C + 63) / 64;
    const float* weights = !WEIGHTS ? nullptr : apart ? sel.weights + (int64_t)b * p.Nk : p.log_weights + b * p.log_weights_batch;
    // Whether points are left out.  dq: only then do the streamed blocks pass through the warp that clears rows.  Either side all of whose points are left out
    // gets zeros at once.
    const int64_t weight_row0 = (p.log_weights_batch == 0 && sel.taken == nullptr ? 0 : (int64_t)b) * ((p.Nk + BLOCK - 1) / BLOCK);       // the first of its blocks
    bool clearing = false;
    if (WEIGHTS) {
        int gone_here = 0, present = 0;
        if (DKDV) {
            if (tid < TILE && row0 + tid < N) present = !(weights[row0 + tid] <= EXCLUDED);
        } else if (apart) {
            present = count > 0;
        } else {
            for (int i = tid; i < count; i += BWD_THREADS) {
                const uint2 gone = stats.gone[weight_row0 + begin + i];
                const int left = M - (begin + i) * BLOCK;
                const uint32_t low = left >= 32 ? ~0u : (1u << left) - 1u, high = left >= 64 ? ~0u : left <= 32 ? 0u : (1u << (left - 32)) - 1u;
                gone_here |= (gone.x | gone.y) != 0;
                present |= ((~gone.x & low) | (~gone.y & high)) != 0;
            }
        }
        if (!DKDV) clearing = __syncthreads_or(gone_here) != 0;
        if (__syncthreads_or(present) == 0) {
            const int chunks = p.C / 8;
            for (int e = tid; e < TILE * chunks; e += BWD_THREADS) {
                const int r = e / chunks, c = (e - r * chunks) * 8, row = row0 + r;
                if (row >= N) continue;
#pragma unroll
                for (int which = 0; which < (DKDV ? 2 : 1); ++which) {
                    if (piece.parts > 1) {
                        const int64_t rest = cut.rest() * TILE;
                        float4* to = reinterpret_cast<float4*>(partials + (which * piece.parts * rest + piece.part * rest + piece.local * TILE + r) * p.C + c);
                        to[0] = to[1] = make_float4(0.f, 0.f, 0.f, 0.f);
                    } else {
                        const View& v = DKDV ? (which == 0 ? p.dk : p.dv) : p.dq;
                        *reinterpret_cast<uint4*>(static_cast<T*>(v.data) + b * v.batch + head * v.head + row * v.point + c) = make_uint4(0, 0, 0, 0);       // (in place: not apart)
                    }
                }
            }
            return;
        }
    }
    auto bar = [&](int i) { return s32(&bars[i]); };
    auto stage = [&](int st) { return s32(base) + K::A_BYTES + st * K::STAGE_BYTES; };

    if (tid == 0) {
        for (int i = 0; i < K::COUNT; ++i) mb_init(bar(i), i == K::A_READY ? (K::A_IN_TMEM ? 16 : WEIGHTS ? 5 : 4) : i >= K::S_DONE && i < K::ACC_DONE ? 8 : i == K::ACC_DONE || (DKDV && i >= K::FREE && i < K::S_FULL) ? 2 : 1);
        fail_s = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s32(&tmem_s)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (EXTRA) {
        // ones (the tile of S for dk, dv gets its rows' weights later), and zeros behind them
        for (int e = tid; e < K::EXTRAS * K::EXTRA_A / 16; e += BWD_THREADS)
            *reinterpret_cast<uint4*>(base + K::OFF_XA + e * 16) = (e & 8) ? make_uint4(0, 0, 0, 0) : make_uint4(EXTRA_ONES_0, EXTRA_ONES_1, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    tm_before();
    __syncthreads();
    tm_after();
    const uint32_t tm = tmem_s;
    bool ok = true;

    if (warp >= 16) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 16 && elect_one()) {
            const CUtensorMap *a1 = apart ? &maps.k_sel_tile : &maps.k_tile, *a2 = apart ? &maps.v_sel_tile : &maps.v_tile;       // (dk, dv)
            const CUtensorMap *b1 = DKDV ? &maps.q : apart ? &maps.k_sel : &maps.k, *b2 = DKDV ? &maps.dout : apart ? &maps.v_sel : &maps.v;
            // ---------------------------------------------------------------- TMA
            if (!K::A_IN_TMEM) {
                mb_expect(bar(K::A_FULL), 2 * slabs * SLAB);
                for (int s = 0; s < slabs; ++s) {
                    tma_load(s32(base) + s * SLAB, a1, s * 64, row0, head, b, bar(K::A_FULL));
                    tma_load(s32(base) + (K::SLABS + s) * SLAB, a2, s * 64, row0, head, b, bar(K::A_FULL));
                }
            }
            int it = 0;
            for (; it < count; ++it) {
                const int st = it % K::STAGES, turn = it / K::STAGES;
                if (turn > 0) ok = mb_wait(bar(K::FREE + st), (turn - 1) & 1, ok);
                if (!ok) break;
                const int g = DKDV ? (begin + it) / per_head : 0, point = (begin + it - g * per_head) * BLOCK, h = DKDV ? head * p.G + g : hk;
                mb_expect(bar(K::FULL + st), 2 * slabs * BSLAB + (EXTRA ? K::EXTRAS * K::EXTRA_B : 0));
                if (DKDV)
                    bulk_load(s32(base) + K::OFF_XB + st * 2 * K::EXTRA_B, stats.extra + (((int64_t)b * p.Hq + h) * per_head + point / BLOCK) * 2 * BLOCK, 2 * K::EXTRA_B, bar(K::FULL + st));
                else if (EXTRA)
                    bulk_load(s32(base) + K::OFF_XB + st * K::EXTRA_B, stats.weights + (weight_row0 + point / BLOCK) * BLOCK, K::EXTRA_B, bar(K::FULL + st));
                for (int s = 0; s < slabs; ++s) {
                    tma_load(stage(st) + s * BSLAB, b1, s * 64, point, h, b, bar(K::FULL + st));
                    tma_load(stage(st) + (K::SLABS + s) * BSLAB, b2, s * 64, point, h, b, bar(K::FULL + st));
                }
            }
            // the copies under way (all there already if all went well)
            if (!K::A_IN_TMEM) mb_wait(bar(K::A_FULL), 0, true);
            for (int i = max(0, it - K::STAGES); i < it; ++i) mb_wait(bar(K::FULL + i % K::STAGES), (i / K::STAGES) & 1, true);
        } else if ((warp == 17 || warp == 19) && elect_one()) {
            // ---------------------------------------------------------------- MMAs: warp 17 S and dv, warp 19 T and dq or dk
            const int which = warp == 17 ? 0 : 1;
            const uint32_t ids = idesc<T>(BLOCK, false), ido = idesc<T>(steps * 16, true), idw = idesc<__nv_bfloat16>(BLOCK, false);
            const uint32_t da = desc_channels(s32(base) + which * K::SLABS * SLAB), db = desc_channels(stage(0) + which * K::SLABS * BSLAB);
            const uint32_t dp = desc_points(stage(0) + (which == 0 ? K::SLABS * BSLAB : 0), BSLAB), ta = tm + K::T_A + which * (D / 2);
            const uint32_t dxa = desc_extra(s32(base) + K::OFF_XA + which * K::EXTRA_A);
            const uint32_t dxb = desc_dense(s32(base) + K::OFF_XB + which * K::EXTRA_B);
            const bool sums = DKDV || which == 1, extra = EXTRA && which < K::EXTRAS;
            const int done = (which == 0 ? K::S_DONE : K::D_READY), full = (which == 0 ? K::S_FULL : K::T_FULL);
            auto first = [&](int it) {
                const int st = it % K::STAGES;
                if (!mb_wait(bar((clearing ? K::READY : K::FULL) + st), (it / K::STAGES) & 1, true)) return false;
                const uint32_t to = tm + K::T_BUF + (it & 1) * 2 * BLOCK + which * BLOCK, bd = db + st * (K::STAGE_BYTES >> 4);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    if (ks < steps) {
                        if constexpr (K::A_IN_TMEM) mma_ts(to, ta + ks * 8, bd + (ks >> 2) * (BSLAB >> 4) + (ks & 3) * 2, ids, ks > 0);
                        else mma_ss(to, da + (ks >> 2) * (SLAB >> 4) + (ks & 3) * 2, bd + (ks >> 2) * (BSLAB >> 4) + (ks & 3) * 2, ids, ks > 0);
                    }
                if (extra) mma_ss<DESC_EXTRA_HIGH, DESC_DENSE_HIGH>(to, dxa, dxb + st * (K::EXTRAS * K::EXTRA_B >> 4), idw, 1);
                mma_commit(bar(full + (it & 1)));
                return true;
            };
            ok = mb_wait(bar(K::A_READY), 0, true) && (K::A_IN_TMEM || mb_wait(bar(K::A_FULL), 0, true));
            tm_after();
            for (int it = 0; it < 2 && it < count && ok; ++it) ok = first(it);
            for (int it = 0; it < count && ok; ++it) {
                ok = mb_wait(bar(done + (it & 1)), (it >> 1) & 1, true);
                if (!ok) break;
                tm_after();
                if (sums) {
                    const int st = it % K::STAGES;
                    const uint32_t at = dp + st * (K::STAGE_BYTES >> 4), from = tm + K::T_BUF + (it & 1) * 2 * BLOCK + which * BLOCK, to = tm + K::T_ACC + (which == 0 ? D : 0);
#pragma unroll
                    for (int kk = 0; kk < BLOCK / 16; ++kk) {
                        const uint32_t a = from + (kk >> 1) * 32 + (kk & 1) * 8;
                        mma_ts(to, a, at + kk * (2048 >> 4), ido, it > 0 || kk > 0);
                        if (FINE) mma_ts(to, a + 16, at + kk * (2048 >> 4), ido, 1);
                    }
                    mma_commit(bar(K::FREE + st));
                }
                if (it + 2 < count) ok = first(it + 2);
            }
            mma_commit(bar(K::ACC_DONE));
            mb_wait(bar(K::ACC_DONE), 0, true);
        } else if (DKDV && WEIGHTS && !K::A_IN_TMEM && warp == 18) {
            // ---------------------------------------------------------------- rows of keys left out
            ok = all_lanes(mb_wait(bar(K::A_FULL), 0, ok));
            for (int r = 0; r < 4 && ok; ++r) {
                const int n = row0 + r * 32 + lane;
                const uint32_t gone = __ballot_sync(0xffffffffu, n < Nk && weight2(weights, n) == -INFINITY);
                for (int which = 0; which < 2; ++which) zero_rows(base + which * K::SLABS * SLAB, slabs, SLAB, r, gone, lane);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mb_arrive(bar(K::A_READY));
        } else if (clearing && warp == 18) {
            // ---------------------------------------------------------------- rows of streamed points left out
            const uint2* gone = stats.gone + weight_row0 + begin;
            uint2 next = gone[0];
            for (int it = 0; it < count && ok; ++it) {
                const int st = it % K::STAGES;
                const uint2 now = next;
                if (it + 1 < count) next = gone[it + 1];
                ok = all_lanes(mb_wait(bar(K::FULL + st), (it / K::STAGES) & 1, ok));
                if (!ok) break;
                if (now.x | now.y) {
                    for (int which = 0; which < 2; ++which) {
                        unsigned char* at = base + K::A_BYTES + st * K::STAGE_BYTES + which * K::SLABS * BSLAB;
                        zero_rows(at, slabs, BSLAB, 0, now.x, lane);
                        zero_rows(at, slabs, BSLAB, 1, now.y, lane);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                __syncwarp();
                if (lane == 0) mb_arrive(bar(K::READY + st));
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int group = (warp >> 2) & 1, half = warp >> 3, row = row0 + (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const bool there = row < N;
        // ---------------------------------------------------------------- operands: group 0 those of S, group 1 those of T, each half its channels
        bool taken = there;         // dk, dv: whether the row's point takes part
        if (DKDV) {
            const float weight = !there ? -INFINITY : WEIGHTS ? weights[row] : 0.f;
            taken = weight > EXCLUDED || weight != weight;
            if (group == 0 && half == 0) {
                const uint2 parts = taken ? extra_parts(weight * (1.f / p.scale)) : make_uint2(EXTRA_OUT, 0);
                *reinterpret_cast<uint4*>(base + K::OFF_XA + extra_at((warp & 3) * 32 + lane)) = make_uint4(parts.x, parts.y | 0x3f800000u, EXTRA_ONES_0, 0);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
        }
        if (K::A_IN_TMEM) {
            const View& v = DKDV ? (group == 0 ? p.k : p.v) : (group == 0 ? p.q : p.dout);
            const int point = !there ? 0 : DKDV && apart ? sel.index[(int64_t)b * p.Nk + row] : row;
            const uint4* from = reinterpret_cast<const uint4*>(static_cast<const T*>(v.data) + b * v.batch + head * v.head + point * v.point);
#pragma unroll
            for (int part = 0; part < D / 64; ++part) {
                const int c = half * (D / 2) + part * 32;
                uint32_t x[16];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 q = taken && c + i * 8 < p.C ? from[c / 8 + i] : make_uint4(0, 0, 0, 0);
                    x[4 * i] = q.x; x[4 * i + 1] = q.y; x[4 * i + 2] = q.z; x[4 * i + 3] = q.w;
                }
                tm_st16(tm + K::T_A + group * (D / 2) + c / 2 + lanes, x);
            }
            tm_st_wait();
        }
        if (K::A_IN_TMEM || (group == 0 && half == 0)) warp_arrive(bar(K::A_READY), lane);
        const float factor = ds_scale<T>(stats, b * p.Hk + hk);
        float neg_lse = 0.f, neg_D = 0.f;       // dq: the row's
        if (!DKDV && there) {
            const int64_t at = ((int64_t)b * p.Hq + head) * p.Nq + row;
            neg_lse = -stats.lse2[at];
            neg_D = -stats.D[at];
        }
        const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2), row_x = pack2(neg_lse, neg_lse), row_D = pack2(neg_D, neg_D), factor2 = pack2(factor, factor);
        const uint32_t from = tm + K::T_BUF + group * 2 * BLOCK + half * 32 + lanes;
        for (int it = group; it < count && ok; it += 2) {
            uint32_t s[32], t[32], x[16], rest[16];
            ok = all_lanes(mb_wait(bar(K::S_FULL + group), (it >> 1) & 1, ok));
            if (!ok) break;
            tm_after();
            tm_ld32(s, from);
            tm_ld_wait();
            if (!DKDV) warp_arrive(bar(K::S_DONE + group), lane);
            if (!DKDV && !WEIGHTS && (begin + it + 1) * BLOCK > M) {
                // points that are not there: zero rows, whose probability must not overflow (the scale is positive)
                const int left = M - (begin + it) * BLOCK - half * 32;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= left) s[i] = 0xff800000u;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint64_t s2 = pack2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), x2 = DKDV ? mul2(s2, scale2) : fma2(s2, scale2, row_x);
                float e0, e1;
                if (i % BY_FMA == BY_FMA - 1) {
                    exp2_by_fma(x2, e0, e1);
                } else {
                    unpack2(x2, e0, e1);
                    e0 = ex2(e0); e1 = ex2(e1);
                }
                s[2 * i] = __float_as_uint(e0);
                s[2 * i + 1] = __float_as_uint(e1);
                if (DKDV) x[i] = pack_parts<T, FINE>(e0, e1, rest[i]);
            }
            if (DKDV) {
                tm_st16(from, x);
                if (FINE) tm_st16(from + 16, rest);
                tm_st_wait();
                warp_arrive(bar(K::S_DONE + group), lane);
            }
            ok = all_lanes(mb_wait(bar(K::T_FULL + group), (it >> 1) & 1, ok));
            if (!ok) break;
            tm_after();
            tm_ld32(t, from + BLOCK);
            tm_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                uint64_t d2 = pack2(__uint_as_float(t[2 * i]), __uint_as_float(t[2 * i + 1]));
                if (!DKDV) d2 = add2(d2, row_D);
                if (SHIFT<T> != 0.f) d2 = mul2(d2, factor2);
                float d0, d1;
                unpack2(mul2(d2, pack2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]))), d0, d1);
                x[i] = pack_parts<T, FINE>(d0, d1, rest[i]);
            }
            tm_st16(from + BLOCK, x);
            if (FINE) tm_st16(from + BLOCK + 16, rest);
            tm_st_wait();
            warp_arrive(bar(K::D_READY + group), lane);
        }
        // ---------------------------------------------------------------- results in pieces of 32 channels: dq by all groups, or dk by group 0 and dv by group 1
        ok = all_lanes(mb_wait(bar(K::ACC_DONE), 0, ok)) && ok;
        if (ok) {
            tm_after();
            const float unshift = ex2(-SHIFT<T>), back = DKDV && group == 1 ? unshift : p.scale * unshift / factor;
            const bool zero = DKDV && !taken;       // (exponentials on the FMA pipe end at 2^-126)
            const View& v = DKDV ? (group == 0 ? p.dk : p.dv) : p.dq;
            const int64_t point = DKDV && apart && there ? sel.index[(int64_t)b * p.Nk + row] : row;
            T* out = static_cast<T*>(v.data) + b * v.batch + head * v.head + point * v.point;
            for (int c = 32 * (DKDV ? half : 2 * half + group); c < p.C; c += DKDV ? 64 : 128) {
                uint32_t o[32];
                tm_ld32(o, tm + K::T_ACC + (DKDV ? group * D : 0) + c + lanes);
                tm_ld_wait();
                if (!there) continue;
                if (piece.parts > 1) {
                    // [dk, dv][part][row][channel]
                    const int64_t rest = cut.rest() * TILE, local = piece.local * TILE + (warp & 3) * 32 + lane;
                    float* to = partials + ((DKDV && group == 1 ? piece.parts * rest : 0) + piece.part * rest + local) * p.C + c;
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        if (c + i < p.C)
                            *reinterpret_cast<float4*>(to + i) = zero ? make_float4(0.f, 0.f, 0.f, 0.f)
                                                                      : make_float4(__uint_as_float(o[i]) * back, __uint_as_float(o[i + 1]) * back, __uint_as_float(o[i + 2]) * back,
                                                                                    __uint_as_float(o[i + 3]) * back);
                    continue;
                }
#pragma unroll
                for (int i = 0; i < 32; i += 8)
                    if (c + i < p.C) {
                        uint32_t y[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) y[k] = zero ? 0u : pack16<T>(__uint_as_float(o[i + 2 * k]) * back, __uint_as_float(o[i + 2 * k + 1]) * back);
                        *reinterpret_cast<uint4*>(out + c + i) = make_uint4(y[0], y[1], y[2], y[3]);
                    }
            }
        }
    }
    if (!ok) atomicExch(&fail_s, 1);
    tm_before();
    __syncthreads();
    if (fail_s && tid == 0) atomicExch(&g_status, 1);
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tm), "r"(512));
}

// One launch for dq and for dk and dv, which need nothing of each other: dq's blocks come first, and the others fill the SMs that its last ones leave idle.
template <typename T, int D, bool WEIGHTS, bool FINE>
__global__ void __launch_bounds__(BWD_THREADS, 1)
attend_backward_tc_kernel(const __grid_constant__ Problem p, const __grid_constant__ Stats stats, const __grid_constant__ Selection sel, const __grid_constant__ BackwardMaps maps,
                          const __grid_constant__ Side dq, const __grid_constant__ Side dkdv) {
    wait_for_previous();        // the statistics
    const int64_t dq_blocks = dq.cut.blocks();
    if (blockIdx.x < dq_blocks) backward_block<T, D, false, WEIGHTS, FINE>(p, stats, sel, maps, dq, blockIdx.x);
    else backward_block<T, D, true, WEIGHTS, FINE>(p, stats, sel, maps, dkdv, blockIdx.x - dq_blocks);
}

// ---- joins of tiles in pieces ---------------------------------------------------------------------------------------------------
//
// A thread takes eight channels of a row; many pieces are shared by up to 32 lanes, whose sums a tree joins: the order is fixed.  (One head of 32, 33 queries, 65536
// points, bf16, 148 pieces: forward pass 60 us with one lane.)  forward: out = sum_s 2^(lse2_s - lse2) out_s; backward: plain sums, of dq, dk and dv
// in one launch.
constexpr int JOIN_THREADS = 256;
struct Join {
    View out, rest;             // rest: what rounding takes from out, forward only; its data may be null
    const float* partials;
    Split cut;
    int64_t threads;
    int lanes;                  // a power of two
    int tiles, rows_per_tile, N, H;
    const int *taken, *index;   // dk, dv: the selection's, or null
};
struct Joins {
    Join join[3];
    float* lse;                 // forward
    int C;
};
template <typename T, bool SOFTMAX>
__global__ void __launch_bounds__(JOIN_THREADS) attend_join_tiles_kernel(const __grid_constant__ Joins a) {
    const Join& j = a.join[SOFTMAX ? 0 : blockIdx.y];
    const int C = a.C, chunks = C / 8, parts = j.cut.parts, lanes = j.lanes, lane = threadIdx.x & (lanes - 1);
    const int64_t thread = (int64_t)blockIdx.x * JOIN_THREADS + threadIdx.x;
    if (thread >= j.threads) return;        // (here and below: all lanes of an item)
    const int64_t rest = j.cut.rest() * j.rows_per_tile, index = thread / lanes, local = index / chunks;
    const int c = (int)(index - local * chunks) * 8;
    const uint32_t mates = (lanes == 32 ? ~0u : (1u << lanes) - 1u) << (threadIdx.x & 31 & ~(lanes - 1));
    const int64_t tile = j.cut.full + local / j.rows_per_tile, bh = tile / j.tiles, b = bh / j.H, h = bh - b * j.H;
    int n = (int)(tile - bh * j.tiles) * j.rows_per_tile + (int)(local % j.rows_per_tile);
    wait_for_previous();
    if (n >= j.N) return;
    if (j.taken != nullptr) {
        const int taken = j.taken[b];
        if (n >= taken) return;
        if (taken != j.N) n = j.index[b * j.N + n];
    }
    const float* statistics = j.partials + parts * rest * C + local;
    float top = -INFINITY, total = 0.f;
    if (SOFTMAX) {
#pragma unroll 4
        for (int s = lane; s < parts; s += lanes) top = fmaxf(top, statistics[s * rest]);
        for (int o = lanes >> 1; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(mates, top, o));
    }
    const float base = top == -INFINITY ? 0.f : top;
    float sum[8] = {};
#pragma unroll 4
    for (int s = lane; s < parts; s += lanes) {
        float w = 1.f;
        if (SOFTMAX) {
            w = ex2(statistics[s * rest] - base);
            total += w;
        }
        const float4* from = reinterpret_cast<const float4*>(j.partials + (s * rest + local) * C + c);
        const float4 x = from[0], y = from[1];
        const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = fmaf(w, v[i], sum[i]);
    }
    for (int o = lanes >> 1; o > 0; o >>= 1) {
        if (SOFTMAX) total += __shfl_xor_sync(mates, total, o);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += __shfl_xor_sync(mates, sum[i], o);
    }
    if (lane != 0) return;
    const float factor = !SOFTMAX ? 1.f : total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] *= factor;
    store8<T>(static_cast<T*>(j.out.data) + b * j.out.batch + h * j.out.head + n * j.out.point + c,
              j.rest.data == nullptr ? nullptr : static_cast<T*>(j.rest.data) + b * j.rest.batch + h * j.rest.head + n * j.rest.point + c, sum);
    if (SOFTMAX && c == 0 && a.lse != nullptr) a.lse[bh * j.N + n] = total == 0.f ? -INFINITY : (top + log2f(total)) * LN2;
}
Join join_of(const View& out, const View& rest, const Split& cut, int rows_per_tile, int N, int H, int C, const float* partials, const Selection& sel) {
    int lanes = 1;
    while (lanes < 32 && lanes * 4 < cut.parts) lanes *= 2;
    const int64_t threads = cut.parts > 1 ? cut.rest() * rows_per_tile * (C / 8) * lanes : 0;
    return Join{out, rest, partials, cut, threads, lanes, (N + rows_per_tile - 1) / rows_per_tile, rows_per_tile, N, H, sel.taken, sel.index};
}
template <typename T, bool SOFTMAX>
cudaError_t launch_joins(const Joins& a, cudaStream_t stream) {
    const int64_t most = std::max({a.join[0].threads, a.join[1].threads, a.join[2].threads});
    if (most == 0) return cudaSuccess;
    return launch_dependent(attend_join_tiles_kernel<T, SOFTMAX>, dim3((unsigned)((most + JOIN_THREADS - 1) / JOIN_THREADS), SOFTMAX ? 1 : 3), JOIN_THREADS, 0, stream, a);
}

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                            CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder() {
    static const Encode fn = [] {
        void* symbol = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &symbol, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) symbol = nullptr;
        return reinterpret_cast<Encode>(symbol);
    }();
    return fn;
}

// Opts a kernel in to its shared memory, once per device (`done`: one bit each; a kernel's own).
template <typename K>
cudaError_t allow(K kernel, size_t bytes, std::atomic<uint64_t>& done) {
    int device = -1;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const uint64_t bit = device < 64 ? (uint64_t)1 << device : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <typename T, int D, bool WEIGHTS>
cudaError_t forward_as(const Problem& p, const Selection& sel, const CUtensorMap (&maps)[5], const Split& cut, float* partials, cudaStream_t stream) {
    const int tiles = (p.Nq + 2 * TILE - 1) / (2 * TILE);
    const auto kernel = attend_forward_tc_kernel<T, D, WEIGHTS>;
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow(kernel, Forward<D>::SMEM, allowed);
    if (e != cudaSuccess) return e;
    const bool selected = sel.taken != nullptr;
    if (selected) e = launch_selection(p, sel, stream);
    if (e != cudaSuccess) return e;
    if (selected) {
        e = launch_dependent(kernel, (unsigned)cut.blocks(), FWD_THREADS, Forward<D>::SMEM, stream, p, sel, maps[0], maps[1], maps[2], maps[3], maps[4], tiles, cut, partials);
    } else {
        kernel<<<(unsigned)cut.blocks(), FWD_THREADS, Forward<D>::SMEM, stream>>>(p, sel, maps[0], maps[1], maps[2], maps[3], maps[4], tiles, cut, partials);
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) return e;
    Joins joins{};
    joins.join[0] = join_of(p.out, p.rest, cut, 2 * TILE, p.Nq, p.Hq, p.C, partials, Selection{});
    joins.lse = p.lse;
    joins.C = p.C;
    return launch_joins<T, true>(joins, stream);
}

template <typename T, int D, bool WEIGHTS, bool FINE>
cudaError_t backward_as(const Problem& p, const Stats& s, const Selection& sel, const BackwardMaps& maps, const Side& dq, const Side& dkdv, cudaStream_t stream) {
    constexpr size_t smem = std::max(Backward<D, false>::SMEM, Backward<D, true>::SMEM);
    const auto kernel = attend_backward_tc_kernel<T, D, WEIGHTS, FINE>;
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow(kernel, smem, allowed);
    if (e != cudaSuccess) return e;
    return launch_dependent(kernel, (unsigned)(dq.cut.blocks() + dkdv.cut.blocks()), BWD_THREADS, smem, stream, p, s, sel, maps, dq, dkdv);
}
// Maps of the selected keys and values (untouched and unread without a selection).
bool make_selected(CUtensorMap& k, CUtensorMap& v, const Problem& p, const Selection& sel, sna_dtype_t dtype, int rows) {
    if (sel.taken == nullptr) return true;
    return make_map(&k, selected_view(p, sel.k), dtype, p.C, p.Nk, p.Hk, p.B, rows) && make_map(&v, selected_view(p, sel.v), dtype, p.C, p.Nk, p.Hk, p.B, rows);
}
// Whether p and ds are held in two 16-bit parts: where their rounding is less averaged out than elsewhere.  With one part the gradients' relative errors (norms) are 1.41 to
// 1.47 times those of rounding the result alone, which is what single roundings of as many terms give; narrow heads reach 1.6, and so do a few rows.  The second part
// costs a forward and backward pass 20 % there (us, B = 2, 4 heads of 8, 8192 queries and points, bf16: 596 with one part, 717 with two), small problems less (1024 queries
// and points, B = 1, 4 heads of 32: 31, 33; 33 queries, 9800 points, one head of 32: 94, 108).
bool in_two_parts(const Problem& p) { return p.C <= 16 || rows_of(p) * p.Nk <= (int64_t)1 << 22; }
}  // namespace

bool backward_tc(const Problem& p, const Stats& s, const Selection& sel, sna_dtype_t dtype, int sms, float* dq_partials, float* dkdv_partials, cudaStream_t stream, cudaError_t& e) {
    BackwardMaps maps;
    const bool wide = p.C > 64;
    if (!make_map(&maps.q, p.q, dtype, p.C, p.Nq, p.Hq, p.B, BLOCK) || !make_map(&maps.dout, p.dout, dtype, p.C, p.Nq, p.Hq, p.B, BLOCK) ||
        !make_map(&maps.k, p.k, dtype, p.C, p.Nk, p.Hk, p.B, BLOCK) || !make_map(&maps.v, p.v, dtype, p.C, p.Nk, p.Hk, p.B, BLOCK) ||
        !make_selected(maps.k_sel, maps.v_sel, p, sel, dtype, BLOCK))
        return false;
    if (wide && (!make_map(&maps.k_tile, p.k, dtype, p.C, p.Nk, p.Hk, p.B, TILE) || !make_map(&maps.v_tile, p.v, dtype, p.C, p.Nk, p.Hk, p.B, TILE) ||
                 !make_selected(maps.k_sel_tile, maps.v_sel_tile, p, sel, dtype, TILE)))
        return false;
    const Side dq{split_of(p, Kernel::DQ, sms), (p.Nq + TILE - 1) / TILE, dq_partials}, dkdv{split_of(p, Kernel::DKDV, sms), (p.Nk + TILE - 1) / TILE, dkdv_partials};
    const bool weights = p.log_weights != nullptr;
    auto run = [&](auto t, auto width) {
        using T = decltype(t);
        constexpr int D = decltype(width)::value;
        auto go = [&](auto fine) {
            constexpr bool FINE = decltype(fine)::value;
            return weights ? backward_as<T, D, true, FINE>(p, s, sel, maps, dq, dkdv, stream) : backward_as<T, D, false, FINE>(p, s, sel, maps, dq, dkdv, stream);
        };
        return in_two_parts(p) ? go(std::true_type()) : go(std::false_type());
    };
    using W64 = std::integral_constant<int, 64>;
    using W128 = std::integral_constant<int, 128>;
    if (dtype == SNA_BFLOAT16) e = wide ? run(__nv_bfloat16(), W128()) : run(__nv_bfloat16(), W64());
    else e = wide ? run(__half(), W128()) : run(__half(), W64());
    return true;
}

// Pieces of each of `rest` tiles, where the SMs have a partial wave of them (see Split).
static int pieces(int64_t rest, int64_t streamed, int64_t least, int sms) {
    double best = 0.97;        // of the partial wave: what gains less is not worth a second kernel, nor is a finer cut for a hundredth
    int parts = 1;
    const int64_t most = std::min(streamed / least, std::max<int64_t>(8, sms / rest));        // (few tiles: one piece per SM)
    for (int64_t k = 2; k <= most; ++k) {
        const double wave = (double)((rest * k + sms - 1) / sms) / (double)k + 0.01 * (double)(k < 8 ? k : 8);
        if (wave < best) { best = wave; parts = (int)k; }
    }
    return parts;
}

Split split_of(const Problem& p, Kernel kernel, int sms) {
    auto up = [](int64_t n, int64_t d) { return (n + d - 1) / d; };
    const int64_t forward = (int64_t)p.B * p.Hq * up(p.Nq, 2 * TILE), dq = (int64_t)p.B * p.Hq * up(p.Nq, TILE), dkdv = (int64_t)p.B * p.Hk * up(p.Nk, TILE);
    const int64_t keys = up(p.Nk, BLOCK), queries = p.G * up(p.Nq, BLOCK);
    // dq's and dk/dv's blocks run side by side, so theirs is one last wave, dk's and dv's; dq is cut if both together are less than a wave, or for its length (below)
    const int64_t tiles = kernel == Kernel::FORWARD ? forward : kernel == Kernel::DQ ? dq : dkdv, all = kernel == Kernel::FORWARD ? forward : dq + dkdv;
    if (kernel == Kernel::DQ || (kernel == Kernel::DKDV && all >= 8 * (int64_t)sms)) {
        // Few queries and many points, or the reverse: what one side's tiles walk is longer than an SM's share of the work, in blocks (a tile's start and end take as long
        // as about ten), dk's and dv's of what is left when they start.  Its tiles are cut to that (dk's and dv's in a few waves are cut below anyway).  (us, backward, bf16: 33
        // queries, 9800 points, one head of 32, tiles whole 81, cut 12; B = 2, 17 queries, 60000 points, 8 and 2 heads of 64 498, 210; 60000 queries, 64 points, 16 heads of 64
        // 852, 543.)
        const bool is_dq = kernel == Kernel::DQ;
        const int64_t length = is_dq ? keys : queries, other = is_dq ? queries : keys, ends = 10;
        const int64_t share = std::max<int64_t>(1, ((is_dq ? dq * (keys + ends) : 0) + dkdv * (queries + ends)) / sms);
        const int64_t parts = std::min(length / 4, up(length, std::max<int64_t>(4, share - ends)));
        if (length > 2 * other && length + ends > 2 * share && parts > 1) return Split{tiles, 0, (int)parts};
    }
    const int64_t rest = std::min(all % sms, tiles);
    Split cut{tiles, tiles, 1};
    if (rest == 0 || all >= 8 * (int64_t)sms || (kernel == Kernel::DQ && all >= sms)) return cut;
    const int parts = kernel == Kernel::FORWARD ? pieces(rest, up(p.Nk, TILE), 2, sms) : pieces(all < sms ? all : rest, all < sms ? std::min(keys, queries) : queries, 4, sms);
    if (parts > 1) cut = Split{tiles, tiles - rest, parts};
    return cut;
}

cudaError_t join_backward(const Problem& p, const Selection& sel, sna_dtype_t dtype, int sms, const float* dq_partials, const float* dkdv_partials, cudaStream_t stream) {
    const Split q = split_of(p, Kernel::DQ, sms), k = split_of(p, Kernel::DKDV, sms);
    Joins joins{};
    joins.join[0] = join_of(p.dq, View{}, q, TILE, p.Nq, p.Hq, p.C, dq_partials, Selection{});
    joins.join[1] = join_of(p.dk, View{}, k, TILE, p.Nk, p.Hk, p.C, dkdv_partials, sel);
    joins.join[2] = join_of(p.dv, View{}, k, TILE, p.Nk, p.Hk, p.C, dkdv_partials + k.parts * k.rest() * TILE * p.C, sel);
    joins.C = p.C;
    return dtype == SNA_BFLOAT16 ? launch_joins<__nv_bfloat16, false>(joins, stream) : launch_joins<__half, false>(joins, stream);
}

size_t partial_floats(const Problem& p, Kernel kernel, int sms) {
    const Split cut = split_of(p, kernel, sms);
    const size_t rows = (size_t)cut.rest() * cut.parts * TILE;
    return kernel == Kernel::FORWARD ? rows * 2 * (p.C + 1) : rows * p.C * (kernel == Kernel::DKDV ? 2 : 1);
}

bool make_map(CUtensorMap* map, const View& v, sna_dtype_t dtype, int C, int N, int H, int B, int rows) {
    const Encode fn = encoder();
    if (fn == nullptr) return false;
    // (a dimension of one is never stepped over: any stride that the driver accepts will do)
    auto bytes = [](int64_t stride, int size) { return (cuuint64_t)(size > 1 ? stride * 2 : 16); };
    const cuuint64_t dims[4] = {(cuuint64_t)C, (cuuint64_t)N, (cuuint64_t)H, (cuuint64_t)B};
    const cuuint64_t strides[3] = {bytes(v.point, N), bytes(v.head, H), bytes(v.batch, B)};
    const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, steps[4] = {1, 1, 1, 1};
    return fn(map, dtype == SNA_BFLOAT16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, v.data, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool forward_tc(const Problem& p, const Selection& sel, sna_dtype_t dtype, int sms, float* partials, cudaStream_t stream, cudaError_t& e) {
    const Split cut = split_of(p, Kernel::FORWARD, sms);
    CUtensorMap maps[5];        // queries, keys, values, the selected keys and values
    if (!make_map(&maps[0], p.q, dtype, p.C, p.Nq, p.Hq, p.B, TILE) || !make_map(&maps[1], p.k, dtype, p.C, p.Nk, p.Hk, p.B, TILE) ||
        !make_map(&maps[2], p.v, dtype, p.C, p.Nk, p.Hk, p.B, TILE) || !make_selected(maps[3], maps[4], p, sel, dtype, TILE))
        return false;
    const bool weights = p.log_weights != nullptr;
    auto run = [&](auto t, auto width) {
        using T = decltype(t);
        constexpr int D = decltype(width)::value;
        return weights ? forward_as<T, D, true>(p, sel, maps, cut, partials, stream) : forward_as<T, D, false>(p, sel, maps, cut, partials, stream);
    };
    using W64 = std::integral_constant<int, 64>;
    using W128 = std::integral_constant<int, 128>;
    if (dtype == SNA_BFLOAT16) e = p.C <= 64 ? run(__nv_bfloat16(), W64()) : run(__nv_bfloat16(), W128());
    else e = p.C <= 64 ? run(__half(), W64()) : run(__half(), W128());
    return true;
}

// A wait on a barrier that nothing arrives on, as long as waits are after one that has run out.
__global__ void wait_probe_kernel() {
    __shared__ unsigned long long bar;
    mb_init(s32(&bar), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (!mb_wait(s32(&bar), 0, false)) atomicExch(&g_status, 1);
}
cudaError_t launch_wait_probe(cudaStream_t stream) {
    wait_probe_kernel<<<1, 1, 0, stream>>>();
    return cudaGetLastError();
}

cudaError_t read_status(int* status) {
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(status, g_status, sizeof(int));
    const int zero = 0;
    if (e == cudaSuccess && *status != 0) e = cudaMemcpyToSymbol(g_status, &zero, sizeof(int));
    return e;
}

}  // namespace attend
}  // namespace sna
