// Eight consecutive elements of a row in one lane: loads, stores and conversions of the types the decode-step calls take.
//
// The kernels of the decode step load through L2 or by ordinary loads, never by __ldg: they start before the kernel in front has
// finished (programmatic dependent launch), what they read may have been written by it, and a non-coherent load may
// return a line that the multiprocessor's L1 holds from before.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "hora_common.cuh"

namespace hora {

struct E4M3 {          // one code; only ever moved eight at a time
    uint8_t bits;
};

template <typename T> struct Raw8;                       // eight elements as they lie in memory
template <> struct Raw8<float> { float4 a, b; };
template <> struct Raw8<__nv_bfloat16> { uint4 a; };
template <> struct Raw8<__half> { uint4 a; };
template <> struct Raw8<E4M3> { uint2 a; };

__device__ __forceinline__ void zero8(Raw8<float> &r) { r.a = r.b = make_float4(0.f, 0.f, 0.f, 0.f); }
__device__ __forceinline__ void zero8(Raw8<__nv_bfloat16> &r) { r.a = make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ void zero8(Raw8<__half> &r) { r.a = make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ void zero8(Raw8<E4M3> &r) { r.a = make_uint2(0, 0); }

__device__ __forceinline__ void load8(Raw8<float> &r, const float *p) {
    r.a = __ldcs(reinterpret_cast<const float4 *>(p));
    r.b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
}
__device__ __forceinline__ void load8(Raw8<__nv_bfloat16> &r, const __nv_bfloat16 *p) { r.a = __ldcs(reinterpret_cast<const uint4 *>(p)); }
__device__ __forceinline__ void load8(Raw8<__half> &r, const __half *p) { r.a = __ldcs(reinterpret_cast<const uint4 *>(p)); }
__device__ __forceinline__ void load8(Raw8<E4M3> &r, const E4M3 *p) { r.a = __ldcs(reinterpret_cast<const uint2 *>(p)); }

__device__ __forceinline__ void store8(const Raw8<float> &r, float *p) {
    reinterpret_cast<float4 *>(p)[0] = r.a;
    reinterpret_cast<float4 *>(p)[1] = r.b;
}
__device__ __forceinline__ void store8(const Raw8<__nv_bfloat16> &r, __nv_bfloat16 *p) { *reinterpret_cast<uint4 *>(p) = r.a; }
__device__ __forceinline__ void store8(const Raw8<__half> &r, __half *p) { *reinterpret_cast<uint4 *>(p) = r.a; }
__device__ __forceinline__ void store8(const Raw8<E4M3> &r, E4M3 *p) { *reinterpret_cast<uint2 *>(p) = r.a; }

__device__ __forceinline__ void widen8(const Raw8<float> &r, float (&x)[8]) {
    x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w;
    x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}
__device__ __forceinline__ void widen8(const Raw8<__nv_bfloat16> &r, float (&x)[8]) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ float2 half2_bits(uint32_t w) {
    __half2 h;
    memcpy(&h, &w, 4);
    return __half22float2(h);
}
__device__ __forceinline__ void widen8(const Raw8<__half> &r, float (&x)[8]) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = half2_bits(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
// Largest magnitude of the eight, by their bits, which order like the magnitudes (infinity and NaN above all others).
__device__ __forceinline__ float largest8(const Raw8<float> &r) {
    const float x[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    return __uint_as_float(m);
}
__device__ __forceinline__ uint32_t largest_half_bits(const uint4 &w) {
    const uint32_t m = __vmaxu2(__vmaxu2(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu), __vmaxu2(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu));
    return max(m & 0xFFFFu, m >> 16);
}
__device__ __forceinline__ float largest8(const Raw8<__nv_bfloat16> &r) { return __uint_as_float(largest_half_bits(r.a) << 16); }
__device__ __forceinline__ float largest8(const Raw8<__half> &r) { return half2_bits(largest_half_bits(r.a)).x; }

// two codes (the low 16 bits) as a pair of halves; exact, NaN stays NaN
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
__device__ __forceinline__ void widen8(const Raw8<E4M3> &r, float (&x)[8]) {
    const uint32_t w[2] = {r.a.x, r.a.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = half2_bits(e4m3x2_to_half2((w[i >> 1] >> (16 * (i & 1))) & 0xFFFFu));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

// round to nearest even
__device__ __forceinline__ void narrow8(const float (&x)[8], Raw8<float> &r) {
    r.a = make_float4(x[0], x[1], x[2], x[3]);
    r.b = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half) {
    const __half2 h = __floats2half2_rn(lo, hi);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack2(x[0], x[1], T()), pack2(x[2], x[3], T()), pack2(x[4], x[5], T()), pack2(x[6], x[7], T()));
}
__device__ __forceinline__ void narrow8(const float (&x)[8], Raw8<__nv_bfloat16> &r) { r.a = pack8<__nv_bfloat16>(x); }
__device__ __forceinline__ void narrow8(const float (&x)[8], Raw8<__half> &r) { r.a = pack8<__half>(x); }
// +-infinity becomes +-448
__device__ __forceinline__ void narrow8(const float (&x)[8], Raw8<E4M3> &r) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * i], x[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        w[i >> 1] |= two << (16 * (i & 1));
    }
    r.a = make_uint2(w[0], w[1]);
}

inline int dtype_bytes(int32_t d) {
    switch (d) {
        case HORA_DTYPE_F32: return 4;
        case HORA_DTYPE_BF16: return 2;
        case HORA_DTYPE_F16: return 2;
        case HORA_DTYPE_E4M3: return 1;
    }
    return 0;
}

// What every call that touches the paged cache checks of it.
inline bool cache_ok(const void *k, const void *v, const void *k_exp, const void *v_exp, int32_t dtype, int64_t n_pages,
                     int32_t page_size, int32_t H, int32_t D) {
    if (dtype != HORA_DTYPE_BF16 && dtype != HORA_DTYPE_F16 && dtype != HORA_DTYPE_E4M3) return false;
    if (H < 1 || (D != 64 && D != 128) || n_pages < 1 || n_pages > 0x7FFFFFFF) return false;
    if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128) return false;
    if (k == nullptr || v == nullptr || ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u)) return false;
    if (dtype == HORA_DTYPE_E4M3) {
        if (k_exp == nullptr || v_exp == nullptr) return false;
        if ((reinterpret_cast<uintptr_t>(k_exp) | reinterpret_cast<uintptr_t>(v_exp)) & 15u) return false;
    }
    return true;
}

}  // namespace hora
