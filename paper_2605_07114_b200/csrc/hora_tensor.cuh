// What the kernels on the tensor cores' own memory (tcgen05) share: barriers in shared memory, copies by TMA, operands, products, loads and
// stores of tensor memory, and pairs of fp32 operations.
#pragma once

#include <cuda.h>

#include <atomic>

#include "hora_checked.cuh"

namespace hora {

constexpr uint32_t kWaitTries = 4000000;                 // a fraction of a second and more; what is waited for takes microseconds

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Waits for the phase of the given parity to complete; false when the limit is reached or another wait of the CTA has failed.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int32_t *failed) {
#pragma unroll 1
    for (uint32_t i = 0; i < kWaitTries; ++i) {
        uint32_t done;
        asm volatile(
            "{\n.reg .pred p;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
            "selp.b32 %0, 1, 0, p;\n}"
            : "=r"(done)
            : "r"(bar), "r"(parity), "r"(1000u)
            : "memory");
        if (done) return true;
        if (*failed) return false;
    }
    *failed = 1;
    (void)HORA_IN(-1, 1);
    return false;
}

__device__ __forceinline__ void tma_box(uint32_t to, const CUtensorMap *map, int32_t x, int32_t y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map),
                 "r"(x), "r"(y), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void tma_box3(uint32_t to, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to), "l"(map),
                 "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}

// Operand in shared memory, 128-byte swizzle.  `lead`: distance between blocks of 64 elements along the contiguous
// direction (used when that is the direction of the rows or columns of the product), groups of eight lie 1024 bytes apart.
// The low word; the high one is the same for all.
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t lead) { return ((at & 0x3FFFFu) >> 4) | ((lead >> 4) << 16); }
constexpr uint32_t kOperandHigh = (1024u >> 4) | (1u << 14) | (2u << 29);

__device__ __forceinline__ void mma_smem(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 da, db;\nmov.b64 da, {%1, %5};\nmov.b64 db, {%2, %5};\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(kOperandHigh)
        : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 db;\nmov.b64 db, {%2, %5};\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(kOperandHigh)
        : "memory");
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0;
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// The same by whole warps, one lane of which (`lead`) is to issue: without a branch, so that what an instruction takes from
// uniform registers is worked out there.
__device__ __forceinline__ void mma_smem(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n.reg .pred p, l;\n.reg .b64 da, db;\nmov.b64 da, {%1, %5};\nmov.b64 db, {%2, %5};\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 l, %6, 0;\n"
        "@l tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(kOperandHigh), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n.reg .pred p, l;\n.reg .b64 db;\nmov.b64 db, {%2, %5};\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 l, %6, 0;\n"
        "@l tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(kOperandHigh), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t lead, uint32_t bar) {
    asm volatile("{\n.reg .pred l;\nsetp.ne.b32 l, %1, 0;\n@l tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"(lead) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of tensor memory, the warp's 32 lanes: one row of them to a thread.
__device__ __forceinline__ void tmem_load(uint32_t at, float (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
          "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]),
          "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]),
          "=f"(r[30]), "=f"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
          "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
        : "r"(at));
}
__device__ __forceinline__ void tmem_store8(uint32_t at, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
                 "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const float (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"f"(r[0]), "f"(r[1]),
        "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "f"(r[8]), "f"(r[9]), "f"(r[10]), "f"(r[11]), "f"(r[12]), "f"(r[13]),
        "f"(r[14]), "f"(r[15]), "r"(at)
        : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two fp32 operations an instruction.
__device__ __forceinline__ uint64_t two(float2 x) { return (uint64_t)__float_as_uint(x.y) << 32 | __float_as_uint(x.x); }
__device__ __forceinline__ float2 two(uint64_t x) { return make_float2(__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32))); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(two(a)), "l"(two(b)), "l"(two(c)));
    return two(d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(two(a)), "l"(two(b)));
    return two(d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(two(a)), "l"(two(b)));
    return two(d);
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// 2^x by multiplications, for x <= 8: the special function unit takes 8 cycles a warp, as long as the tensor cores need for its
// share of the products, so a quarter of the exponentials is computed beside it.  2^x = 2^n 2^f, n = round(x), |f| <= 1/2;
// 2^f by the polynomial of degree 5 with the least largest relative error (7.5e-8, 2.0e-7 with fp32 rounding; fitted by iterated
// weighted least squares), times 2^n, whose exponent comes from the low bits of the rounding.  Below 2^-126.5, for the -infinity of a hidden
// key too, 2^n is 0 and so is the result, as the special function unit has it; NaN stays NaN.
__device__ __forceinline__ float2 exp2_by_products(float2 x) {
    x = make_float2(max_or_nan(x.x, -127.f), max_or_nan(x.y, -127.f));
    const float2 big = make_float2(12582912.f, 12582912.f), t = add2(x, big);      // 1.5 * 2^23: the low bits of t are n
    const float2 f = fma2(add2(t, make_float2(-12582912.f, -12582912.f)), make_float2(-1.f, -1.f), x);
    float2 p = make_float2(1.3276471519402e-3f, 1.3276471519402e-3f);
    p = fma2(p, f, make_float2(9.6755413306768e-3f, 9.6755413306768e-3f));
    p = fma2(p, f, make_float2(5.5507132749614e-2f, 5.5507132749614e-2f));
    p = fma2(p, f, make_float2(2.4022119723934e-1f, 2.4022119723934e-1f));
    p = fma2(p, f, make_float2(6.9314696706386e-1f, 6.9314696706386e-1f));
    p = fma2(p, f, make_float2(1.0000000716547f, 1.0000000716547f));
    return mul2(p, make_float2(__uint_as_float((__float_as_uint(t.x) << 23) + 0x3F800000u), __uint_as_float((__float_as_uint(t.y) << 23) + 0x3F800000u)));
}

// ---- host

using TensorMapEncode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                     const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
TensorMapEncode tensor_map_encode();                     // cuTensorMapEncodeTiled, or null

// Rows of heads as [tokens][H][D], `row_stride` elements from token to token, fetched 64 elements of box_h heads of box_t tokens at a time;
// what is beyond the last token comes as zeros.
bool head_map(CUtensorMap *map, const void *rows, int32_t dtype, int32_t D, int32_t H, int64_t tokens, int64_t row_stride, int32_t box_h, int32_t box_t);

// Shared memory beyond the default has to be asked for once per kernel and device.
cudaError_t allow_shared(const void *kernel, int bytes, std::atomic<uint64_t> &devices);

}  // namespace hora
