// tcgen05, TMEM, TMA and mbarrier primitives of the 16-bit attention's large kernels.
#pragma once
#include <cuda.h>

#include "sna_attend.cuh"

namespace sna {
namespace attend {

constexpr int WAIT_POLLS = 1 << 17;     // of one wait (each may suspend for up to ~2 us) before the thread gives up

__device__ __forceinline__ uint32_t s32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// One lane of a whole warp, in a form from which the compiler knows that one lane is left (MMAs then issue back to back).
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}\n" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void mb_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void mb_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void mb_expect(uint32_t bar, uint32_t bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ bool mb_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
                 : "=r"(done) : "r"(bar), "r"(parity), "r"(2000u) : "memory");
    return done != 0;
}
// Bounded wait; once one has run out (`healthy` false) later ones give up at once.
__device__ __forceinline__ bool mb_wait(uint32_t bar, uint32_t parity, bool healthy) {
    if (mb_try(bar, parity)) return true;
    bool done = false;
    const int limit = healthy ? WAIT_POLLS : 4;
    for (int it = 0; it < limit && !done; ++it) done = mb_try(bar, parity);
    return done;
}
// [channel, point, head, batch]: 64 channels (128 bytes) of the map's rows, 128-byte swizzle
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int c, int point, int head, int batch, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(c), "r"(point), "r"(head), "r"(batch), "r"(bar) : "memory");
}

// Shared-memory operands: rows (points) of 128 bytes (64 channels), groups of 8 rows 1024 bytes apart, 128-byte swizzle; a second slab holds
// the channels from 64.  The same tile serves a sum over channels (K-major: a step of 16 channels is 32 bytes further) and, as a B operand
// whose columns are channels, a sum over points (MN-major: a step of 16 points is 2048 bytes further, the next 64 channels a slab).
// A descriptor is held as its low half, which addresses (in units of 16 bytes) move along; the high half is the same for all of these tiles.
constexpr uint32_t DESC_HIGH = (1024 >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_channels(uint32_t addr) { return (addr >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_points(uint32_t addr, uint32_t slab) { return (addr >> 4) | ((slab >> 4) << 16); }
// Rows of 16 bytes without a swizzle, 8 rows 256 bytes apart, and a second half of a step's 16 channels 128 bytes further: one step of extra channels
// beside a tile, that add a number per point to the scores (the number in three bfloat16 parts against ones: 24 bits).
constexpr uint32_t DESC_EXTRA_HIGH = (256 >> 4) | (1u << 14);
__device__ __forceinline__ uint32_t desc_extra(uint32_t addr) { return (addr >> 4) | ((128u >> 4) << 16); }
__device__ __forceinline__ int extra_at(int row) { return (row >> 3) * 256 + (row & 7) * 16; }
// The same as a B operand without the second half: 8 rows 128 bytes apart, and the first half read in its place (against zeros).
constexpr uint32_t DESC_DENSE_HIGH = (128 >> 4) | (1u << 14);
__device__ __forceinline__ uint32_t desc_dense(uint32_t addr) { return addr >> 4; }

// fp32 accumulator, both operands T, 128 rows, n columns
template <typename T> __device__ __forceinline__ uint32_t idesc(int n, bool b_is_points) {
    const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
    return (1u << 4) | (type << 7) | (type << 10) | ((b_is_points ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
template <uint32_t HIGH_A = DESC_HIGH, uint32_t HIGH_B = HIGH_A>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %6};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}\n" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"(HIGH_A), "n"(HIGH_B) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}\n" ::"r"(d), "r"(a_tmem), "r"(b), "r"(idesc), "r"(acc), "n"(DESC_HIGH) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tm_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 32 columns of the warp's 32 lanes; the registers are valid after tm_ld_wait()
__device__ __forceinline__ void tm_ld32(uint32_t* r, uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]),"=r"(r[1]),"=r"(r[2]),"=r"(r[3]),"=r"(r[4]),"=r"(r[5]),"=r"(r[6]),"=r"(r[7]),"=r"(r[8]),"=r"(r[9]),"=r"(r[10]),"=r"(r[11]),"=r"(r[12]),"=r"(r[13]),"=r"(r[14]),"=r"(r[15]),
          "=r"(r[16]),"=r"(r[17]),"=r"(r[18]),"=r"(r[19]),"=r"(r[20]),"=r"(r[21]),"=r"(r[22]),"=r"(r[23]),"=r"(r[24]),"=r"(r[25]),"=r"(r[26]),"=r"(r[27]),"=r"(r[28]),"=r"(r[29]),"=r"(r[30]),"=r"(r[31]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_st32(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        :: "r"(addr), "r"(r[0]),"r"(r[1]),"r"(r[2]),"r"(r[3]),"r"(r[4]),"r"(r[5]),"r"(r[6]),"r"(r[7]),"r"(r[8]),"r"(r[9]),"r"(r[10]),"r"(r[11]),"r"(r[12]),"r"(r[13]),"r"(r[14]),"r"(r[15]),
           "r"(r[16]),"r"(r[17]),"r"(r[18]),"r"(r[19]),"r"(r[20]),"r"(r[21]),"r"(r[22]),"r"(r[23]),"r"(r[24]),"r"(r[25]),"r"(r[26]),"r"(r[27]),"r"(r[28]),"r"(r[29]),"r"(r[30]),"r"(r[31]) : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        :: "r"(addr), "r"(r[0]),"r"(r[1]),"r"(r[2]),"r"(r[3]),"r"(r[4]),"r"(r[5]),"r"(r[6]),"r"(r[7]),"r"(r[8]),"r"(r[9]),"r"(r[10]),"r"(r[11]),"r"(r[12]),"r"(r[13]),"r"(r[14]),"r"(r[15]) : "memory");
}
// 2^x for two numbers of at most 2^6 on the FMA pipe, beside the special-function unit that ex2 uses: x = n + f with |f| <= 1/2 (Cody and Waite),
// 2^f by the polynomial of degree 4 with the least relative error there (2.6e-6 = 2^-18.5, found by iterated least squares), times 2^n.  Numbers below -126
// count as -126; NaN stays NaN.
__device__ __forceinline__ void exp2_by_fma(uint64_t x2, float& y0, float& y1) {
    float x0, x1;
    unpack2(x2, x0, x1);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x0) : "f"(-126.f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x1) : "f"(-126.f));
    x2 = pack2(x0, x1);
    const uint64_t round2 = pack2(12582912.f, 12582912.f), back2 = pack2(-12582912.f, -12582912.f), minus2 = pack2(-1.f, -1.f);     // 1.5 * 2^23: n in the low bits
    const uint64_t t2 = add2(x2, round2), f2 = fma2(add2(t2, back2), minus2, x2);
    uint64_t p2 = pack2(0.009570102f, 0.009570102f);
    p2 = fma2(p2, f2, pack2(0.055917863f, 0.055917863f));
    p2 = fma2(p2, f2, pack2(0.24024744f, 0.24024744f));
    p2 = fma2(p2, f2, pack2(0.6931218f, 0.6931218f));
    p2 = fma2(p2, f2, pack2(0.9999993f, 0.9999993f));
    float t0, t1;
    unpack2(t2, t0, t1);
    t0 = __uint_as_float((__float_as_uint(t0) << 23) + 0x3f800000u);
    t1 = __uint_as_float((__float_as_uint(t1) << 23) + 0x3f800000u);
    unpack2(mul2(p2, pack2(t0, t1)), y0, y1);
}
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }

template <typename T> __device__ __forceinline__ uint32_t pack16(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack16<__nv_bfloat16>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t pack16<__half>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// log2 of a point's weight, -infinity if it is left out
__device__ __forceinline__ float weight2(const float* weights, int n) {
    if (weights == nullptr) return 0.f;
    const float w = weights[n];
    return w <= EXCLUDED ? -INFINITY : w * LOG2E;
}

// Makes rows of a tile zero whose point is left out: called by a whole warp, bit `lane` of `gone` for row 32 r + lane of each slab.  A lane
// writes its own row's 16-byte pieces, in an order in which eight lanes meet eight different banks' groups.  The writes are ordered before the
// tensor core's reads by the proxy fence and the arrival that follow.
__device__ __forceinline__ void zero_rows(unsigned char* tile, int slabs, int slab_bytes, int r, uint32_t gone, int lane) {
    if (!((gone >> lane) & 1)) return;
    for (int s = 0; s < slabs; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(tile + s * slab_bytes + (r * 32 + lane) * 128 + ((i + lane) & 7) * 16) = make_uint4(0, 0, 0, 0);
}

// A map over a tensor's [channel, point, head, batch], boxes of 64 channels x `rows` points (sna_kernels_attend_tc.cu); false if the driver refuses.
bool make_map(CUtensorMap* map, const View& v, sna_dtype_t dtype, int C, int N, int H, int B, int rows);

}  // namespace attend
}  // namespace sna
