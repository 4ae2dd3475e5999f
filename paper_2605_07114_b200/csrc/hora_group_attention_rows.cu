// hora_group_attention, the kernel for items of up to 16 query rows: decode of single tokens over long caches.
//
// The call is bound by the cache's bytes (16 rows or fewer to a key: at most 16 products a byte), so the tensor unit matters only in
// that it has to be out of the way, and what counts is loads in flight.  Keys and values go from global memory
// straight into the registers that mma.m16n8k16 takes them in, with no shared memory, no barrier and no copy in between:
//   - scores S = Q K^T sum over the head's dimensions, in any order that Q and K agree on: lane (n, c) = (lane / 4, lane % 4) of
//     a warp takes 16 neighbouring bytes of key n, and the four lanes of a key neighbouring blocks of 16;
//   - O += P V sums over keys, two neighbouring ones to a register: lane (n, c) loads 16 bytes of keys 2c, 2c+1, 2c+8, 2c+9
//     from dimension n * 8 (16 for one-byte values) on and pairs them up by byte permutations.  The column n of the product then is
//     dimension n * 8 + j of the head for the j-th register: a lane ends up with runs of neighbouring dimensions.
// Each warp runs over its own keys with its own running maximum, sum and output; the next keys are requested
// before the softmax of the present ones, the next values after their product.  The four warps of a CTA take a step's 64 keys,
// 16 each, and join their partials in shared memory when the CTA's part of an item ends.
//
// An e4m3 cache is multiplied in fp16, which holds its codes exactly: a row's power-of-two scale is applied to its score, and to
// its weight relative to the largest value scale met so far, so that weights stay within [0, 1]; queries are scaled by a power of
// two to lie well within fp16's range.
#include "hora_group_attention.cuh"

namespace hora {

constexpr int kStepThreads = 128;
constexpr int kStepWarps = kStepThreads / kWarp;
constexpr int kWarpKeys = kStepKeys / kStepWarps;        // 16: one mma's worth
static_assert(kWarpKeys == 16, "a warp takes sixteen keys of a step");

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(kFull, v, 1));
    return fmaxf(v, __shfl_xor_sync(kFull, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
    v += __shfl_xor_sync(kFull, v, 1);
    return v + __shfl_xor_sync(kFull, v, 2);
}

__device__ __forceinline__ float exponent_byte(uint32_t b) { return __uint_as_float(b ? b << 23 : 0x400000u); }

// sixteen keys of a warp on their way through the registers
template <bool F8, int D>
struct Keys {
    static constexpr int kBlocks = F8 ? D / 64 : D / 32;          // 16-byte loads for each key in K
    static constexpr int kHalves = F8 ? 1 : D / 64;               // 16-byte (D = 64 in one-byte values: 8-byte) loads for each key in V
    uint4 k[2][kBlocks], v[4][kHalves];
    uint32_t ke[2], ve[2];                                        // scale bytes of keys 2c, 2c+1 and 2c+8, 2c+9
};

template <typename Q, bool F8, int D>
__global__ void __launch_bounds__(kStepThreads, 3)
attention_rows_kernel(const AttnArgs a) {
    pdl_enter();
    using M = std::conditional_t<F8, __half, Q>;                  // the type of the products
    using Elem = std::conditional_t<F8, uint8_t, uint16_t>;       // a cached element
    constexpr int kBlocks = Keys<F8, D>::kBlocks, kHalves = Keys<F8, D>::kHalves;
    constexpr int kBlockDims = F8 ? 64 : 32;                      // dimensions of one K load over the four lanes of a key
    constexpr int kOut = D / 8;                                   // column tiles of the output
    __shared__ float s_o[kStepWarps][kTileRows][D + 4];
    __shared__ float s_m[kStepWarps][kTileRows], s_l[kStepWarps][kTileRows];
    const int lane = lane_id(), warp = threadIdx.x >> 5;
    const int n = lane >> 2, c = lane & 3;
    const int32_t n_seq = a.N + a.R;
    const int64_t total = __ldg(a.start + n_seq);
    const int64_t per = (total + a.n_ctas - 1) / a.n_ctas;
    const int64_t rows_all = (int64_t)a.R * a.T * a.Hq;
    int64_t u = (int64_t)blockIdx.x * per;
    const int64_t u_end = min(total, u + per);
    if (u >= u_end) return;

    // the sequence that holds step u: the last i with start[i] <= u, 32 probes at a time
    int32_t i = 0;
    for (int32_t lo = 0, hi = n_seq;;) {                          // start[lo] <= u < start[hi]
        const int32_t gap = (hi - lo + kWarp - 1) / kWarp;
        const int32_t probe = min(hi, lo + lane * gap);
        const unsigned at_or_before = __ballot_sync(kFull, __ldg(a.start + probe) <= u && probe < hi);
        const int32_t top = 31 - __clz(at_or_before);             // lane 0 always is
        hi = min(hi, lo + (top + 1) * gap);
        lo = lo + top * gap;
        i = lo;
        if (hi - lo <= 1) break;
    }
    bool bad = false;
    Sequence s = sequence(a, i, bad);
    int64_t s_start = __ldg(a.start + i);

    while (u < u_end) {
        while (u >= s_start + (int64_t)s.steps * s.tiles * a.Hkv) {           // on to the next sequence that has steps
            s_start += (int64_t)s.steps * s.tiles * a.Hkv;
            ++i;
            s = sequence(a, i, bad);
        }
        const int64_t item = (u - s_start) / s.steps;
        const int32_t step0 = (int32_t)((u - s_start) - item * s.steps);
        const int32_t step1 = (int32_t)min((int64_t)s.steps, step0 + (u_end - u));
        const int32_t h = (int32_t)(item / s.tiles), tile = (int32_t)(item % s.tiles);
        const bool prompt = i < a.N;
        const int32_t *__restrict__ pages = prompt ? a.prefix_pages + (int64_t)i * a.prefix_ld
                                                   : a.suffix_pages + (int64_t)(i - a.N) * a.suffix_ld;
        // rows n and n + 8 of the tile are this lane's
        const QueryRow row0 = query_row(a, s, prompt, h, tile * kTileRows + n);
        const QueryRow row1 = query_row(a, s, prompt, h, tile * kTileRows + n + 8);
        uint32_t qf[2 * kBlocks * (F8 ? 2 : 1)][4];               // one mma step (16 dimensions) each
        float q_unit0 = 1.f, q_unit1 = 1.f;                       // what the stored queries have to be multiplied by
        {
            constexpr int kLoads = kBlocks * (F8 ? 2 : 1);
            uint4 x0[kLoads], x1[kLoads];
#pragma unroll
            for (int b = 0; b < kLoads; ++b) {
                const int dim = F8 ? (b >> 1) * 64 + c * 16 + (b & 1) * 8 : b * 32 + c * 8;
                x0[b] = x1[b] = make_uint4(0, 0, 0, 0);
                const Q *__restrict__ q = static_cast<const Q *>(a.q);
                if (row0.out >= 0) x0[b] = __ldg(reinterpret_cast<const uint4 *>(q + row0.out / a.Hq * a.q_row_stride + row0.out % a.Hq * D + dim));
                if (row1.out >= 0) x1[b] = __ldg(reinterpret_cast<const uint4 *>(q + row1.out / a.Hq * a.q_row_stride + row1.out % a.Hq * D + dim));
            }
            if constexpr (F8) {
                // to fp16 with the row's largest value in [64, 128): smaller ones keep 11 bits down to 2^-21 of it
                float m0 = 0.f, m1 = 0.f, y0[kLoads][8], y1[kLoads][8];
#pragma unroll
                for (int b = 0; b < kLoads; ++b) {
                    widen8(Raw8<Q>{x0[b]}, y0[b]);
                    widen8(Raw8<Q>{x1[b]}, y1[b]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) { m0 = fmaxf(m0, fabsf(y0[b][e])); m1 = fmaxf(m1, fabsf(y1[b][e])); }
                }
                auto unit = [](float m) {
                    const int e = (int)(__float_as_uint(m) >> 23) - 127 - 6;
                    return m > 0.f && e < 120 ? __uint_as_float((uint32_t)(max(e, -120) + 127) << 23) : 1.f;
                };
                q_unit0 = unit(quad_max(m0));
                q_unit1 = unit(quad_max(m1));
                const float f0 = 1.f / q_unit0, f1 = 1.f / q_unit1;              // powers of two: exact
#pragma unroll
                for (int b = 0; b < kLoads; ++b) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) { y0[b][e] *= f0; y1[b][e] *= f1; }
                    x0[b] = pack8<__half>(y0[b]);
                    x1[b] = pack8<__half>(y1[b]);
                }
            }
#pragma unroll
            for (int b = 0; b < kLoads; ++b) {
                const uint32_t w0[4] = {x0[b].x, x0[b].y, x0[b].z, x0[b].w}, w1[4] = {x1[b].x, x1[b].y, x1[b].z, x1[b].w};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    qf[2 * b + j][0] = w0[2 * j];
                    qf[2 * b + j][1] = w1[2 * j];
                    qf[2 * b + j][2] = w0[2 * j + 1];
                    qf[2 * b + j][3] = w1[2 * j + 1];
                }
            }
        }
        const float to_log2_0 = a.scale_log2 * q_unit0, to_log2_1 = a.scale_log2 * q_unit1;

        float o[kOut][4] = {};
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float v_unit = 0.f;                                       // F8: o is in units of this (0: nothing added yet)

        Keys<F8, D> x;
        auto page_row = [&](int32_t key) {                        // pool row of the warp's first key; lengths end inside the table
            int32_t p = key < s.len ? __ldg(pages + (key >> a.page_shift)) : 0;
            if (p < 0 || p >= a.n_pages) { bad = true; p = 0; }
            return (((int64_t)p * a.Hkv + h) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
        };
        auto load_k = [&](int64_t row) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
                    x.k[j][b] = __ldcs(reinterpret_cast<const uint4 *>(static_cast<const Elem *>(a.k_cache) + (row + j * 8 + n) * D + b * kBlockDims + c * (16 / (int)sizeof(Elem))));
            if constexpr (F8) {
#pragma unroll
                for (int j = 0; j < 2; ++j) x.ke[j] = __ldg(reinterpret_cast<const uint16_t *>(a.k_exp + row + j * 8 + 2 * c));
            }
        };
        auto load_v = [&](int64_t row) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int b = 0; b < kHalves; ++b) {
                    const Elem *__restrict__ p = static_cast<const Elem *>(a.v_cache) + (row + (j >> 1) * 8 + 2 * c + (j & 1)) * D;
                    if constexpr (F8 && D == 64) {
                        const uint2 y = __ldcs(reinterpret_cast<const uint2 *>(p + n * 8));
                        x.v[j][b] = make_uint4(y.x, y.y, 0u, 0u);
                    } else if constexpr (F8) {
                        x.v[j][b] = __ldcs(reinterpret_cast<const uint4 *>(p + n * 16));
                    } else {
                        x.v[j][b] = __ldcs(reinterpret_cast<const uint4 *>(p + b * 64 + n * 8));
                    }
                }
            if constexpr (F8) {
#pragma unroll
                for (int j = 0; j < 2; ++j) x.ve[j] = __ldg(reinterpret_cast<const uint16_t *>(a.v_exp + row + j * 8 + 2 * c));
            }
        };

        int32_t key = step0 * kStepKeys + warp * kWarpKeys;
        const int32_t key_end = min(step1 * kStepKeys, s.len);
        if (key < key_end) {
            const int64_t row = page_row(key);
            load_k(row);
            load_v(row);
        }
        for (; key < key_end; key += kStepKeys) {
            const int64_t next = key + kStepKeys < key_end ? page_row(key + kStepKeys) : -1;
            float sc[2][4] = {};
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    const uint32_t w[4] = {x.k[j][b].x, x.k[j][b].y, x.k[j][b].z, x.k[j][b].w};
                    if constexpr (F8) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            mma16816(sc[j], qf[4 * b + e], e4m3x2_to_half2(w[e] & 0xFFFFu), e4m3x2_to_half2(w[e] >> 16), M());
                    } else {
                        mma16816(sc[j], qf[2 * b], w[0], w[1], M());
                        mma16816(sc[j], qf[2 * b + 1], w[2], w[3], M());
                    }
                }
            uint32_t ke[2] = {0u, 0u};
            if constexpr (F8) { ke[0] = x.ke[0]; ke[1] = x.ke[1]; }
            if (next >= 0) load_k(next);
            // scores in units of log2, hidden keys at -infinity
            const bool whole = key + kWarpKeys <= min(row0.limit, row1.limit);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float f = e < 2 ? to_log2_0 : to_log2_1;
                    if constexpr (F8) f *= exponent_byte((ke[j] >> (8 * (e & 1))) & 0xFFu);
                    sc[j][e] *= f;
                    if (!whole && key + j * 8 + 2 * c + (e & 1) >= (e < 2 ? row0.limit : row1.limit)) sc[j][e] = -INFINITY;
                }
            const float top0 = fmaxf(m0, quad_max(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[1][0], sc[1][1]))));
            const float top1 = fmaxf(m1, quad_max(fmaxf(fmaxf(sc[0][2], sc[0][3]), fmaxf(sc[1][2], sc[1][3]))));
            // where no key has been seen the maximum is -infinity and every weight has to come out as 0
            const float z0 = top0 == -INFINITY ? 0.f : top0, z1 = top1 == -INFINITY ? 0.f : top1;
            float f0 = exp2f(m0 - z0), f1 = exp2f(m1 - z1);
            m0 = top0;
            m1 = top1;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[j][e] = exp2f(sc[j][e] - (e < 2 ? z0 : z1));
            l0 = l0 * f0 + ((sc[0][0] + sc[0][1]) + (sc[1][0] + sc[1][1]));
            l1 = l1 * f1 + ((sc[0][2] + sc[0][3]) + (sc[1][2] + sc[1][3]));
            if constexpr (F8) {
                float e4[4], top = v_unit;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = key + (j >> 1) * 8 + 2 * c + (j & 1) < s.len;
                    e4[j] = in ? exponent_byte((x.ve[j >> 1] >> (8 * (j & 1))) & 0xFFu) : 0.f;
                    top = fmaxf(top, e4[j]);
                }
                top = quad_max(top);                              // the same in all quads: they hold the same keys
                const float inv = 1.f / top;                      // powers of two; at least one key is within the length
                f0 *= v_unit * inv;
                f1 *= v_unit * inv;
                v_unit = top;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[j][e] *= e4[2 * j + (e & 1)] * inv;
            }
#pragma unroll
            for (int t = 0; t < kOut; ++t) { o[t][0] *= f0; o[t][1] *= f0; o[t][2] *= f1; o[t][3] *= f1; }
            if (key + kWarpKeys > s.len) {                        // what lies beyond the length may be anything: 0 * NaN is not 0
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (key + (j >> 1) * 8 + 2 * c + (j & 1) >= s.len)
#pragma unroll
                        for (int b = 0; b < kHalves; ++b) x.v[j][b] = make_uint4(0, 0, 0, 0);
            }
            const uint32_t p[4] = {pack2(sc[0][0], sc[0][1], M()), pack2(sc[0][2], sc[0][3], M()),
                                   pack2(sc[1][0], sc[1][1], M()), pack2(sc[1][2], sc[1][3], M())};
#pragma unroll
            for (int b = 0; b < kHalves; ++b) {
                const uint32_t v0[4] = {x.v[0][b].x, x.v[0][b].y, x.v[0][b].z, x.v[0][b].w};
                const uint32_t v1[4] = {x.v[1][b].x, x.v[1][b].y, x.v[1][b].z, x.v[1][b].w};
                const uint32_t v2[4] = {x.v[2][b].x, x.v[2][b].y, x.v[2][b].z, x.v[2][b].w};
                const uint32_t v3[4] = {x.v[3][b].x, x.v[3][b].y, x.v[3][b].z, x.v[3][b].w};
                if constexpr (F8) {
#pragma unroll
                    for (int w = 0; w < kOut / 4; ++w) {          // four dimensions of a key to a word
                        const uint32_t lo0 = __byte_perm(v0[w], v1[w], 0x5140), hi0 = __byte_perm(v0[w], v1[w], 0x7362);
                        const uint32_t lo1 = __byte_perm(v2[w], v3[w], 0x5140), hi1 = __byte_perm(v2[w], v3[w], 0x7362);
                        mma16816(o[4 * w], p, e4m3x2_to_half2(lo0 & 0xFFFFu), e4m3x2_to_half2(lo1 & 0xFFFFu), M());
                        mma16816(o[4 * w + 1], p, e4m3x2_to_half2(lo0 >> 16), e4m3x2_to_half2(lo1 >> 16), M());
                        mma16816(o[4 * w + 2], p, e4m3x2_to_half2(hi0 & 0xFFFFu), e4m3x2_to_half2(hi1 & 0xFFFFu), M());
                        mma16816(o[4 * w + 3], p, e4m3x2_to_half2(hi0 >> 16), e4m3x2_to_half2(hi1 >> 16), M());
                    }
                } else {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {                 // two dimensions of a key to a word
                        mma16816(o[8 * b + 2 * w], p, __byte_perm(v0[w], v1[w], 0x5410), __byte_perm(v2[w], v3[w], 0x5410), M());
                        mma16816(o[8 * b + 2 * w + 1], p, __byte_perm(v0[w], v1[w], 0x7632), __byte_perm(v2[w], v3[w], 0x7632), M());
                    }
                }
            }
            if (next >= 0) load_v(next);
        }
        l0 = quad_sum(l0);
        l1 = quad_sum(l1);

        // join the four warps.  o[t] holds columns 2c and 2c+1 of tile t: dimension column * run + t within its part of the head
        constexpr int kRun = F8 ? D / 8 : 8;
#pragma unroll
        for (int t = 0; t < kOut; ++t) {
            const int part = F8 ? 0 : (t >> 3) * 64, j = F8 ? t : t & 7;
            const float f = F8 ? v_unit : 1.f;
            s_o[warp][n][part + 2 * c * kRun + j] = o[t][0] * f;
            s_o[warp][n][part + (2 * c + 1) * kRun + j] = o[t][1] * f;
            s_o[warp][n + 8][part + 2 * c * kRun + j] = o[t][2] * f;
            s_o[warp][n + 8][part + (2 * c + 1) * kRun + j] = o[t][3] * f;
        }
        if (c == 0) {
            s_m[warp][n] = m0;
            s_m[warp][n + 8] = m1;
            s_l[warp][n] = l0;
            s_l[warp][n + 8] = l1;
        }
        __syncthreads();
        const int32_t tile_rows = min(kTileRows, s.rows - tile * kTileRows);
        for (int32_t at = warp; at < tile_rows; at += kStepWarps) {
            float m = -INFINITY, l = 0.f, f[kStepWarps];
#pragma unroll
            for (int w = 0; w < kStepWarps; ++w) m = fmaxf(m, s_m[w][at]);
            const float z = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int w = 0; w < kStepWarps; ++w) {
                f[w] = exp2f(s_m[w][at] - z);
                l += s_l[w][at] * f[w];
            }
            const int64_t out = query_row(a, s, prompt, h, tile * kTileRows + at).out;
            const int64_t place = step0 > 0 ? (int64_t)blockIdx.x * kTileRows + at : (prompt ? out : rows_all + out);
            float *__restrict__ po = (step0 > 0 ? a.cont_o : a.main_o) + place * D;
            float *__restrict__ pml = (step0 > 0 ? a.cont_ml : a.main_ml) + place * 2;
#pragma unroll
            for (int d = lane * 2; d < D; d += 2 * kWarp) {
                float2 y = make_float2(0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kStepWarps; ++w) {
                    const float2 v = *reinterpret_cast<const float2 *>(&s_o[w][at][d]);
                    y.x += v.x * f[w];
                    y.y += v.y * f[w];
                }
                *reinterpret_cast<float2 *>(po + d) = y;
            }
            if (lane == 0) *reinterpret_cast<float2 *>(pml) = make_float2(m, l);
        }
        __syncthreads();
        u += step1 - step0;
    }
    if (bad) raise_status(a.status, HORA_ERR_INVALID_VALUE);
}

hora_status_t launch_attention_steps(const AttnArgs &a, int32_t q_dtype, int32_t cache_dtype, int32_t D, cudaStream_t stream) {
    auto go = [&](auto kernel) {
        const cudaError_t e = launch_pdl(kernel, a.n_ctas, kStepThreads, 0, stream, a);
        count_launches(1);
        return cuda_ok(e);
    };
    const bool bf = q_dtype == HORA_DTYPE_BF16;
    if (cache_dtype == HORA_DTYPE_E4M3) {
        if (D == 64) return bf ? go(attention_rows_kernel<__nv_bfloat16, true, 64>) : go(attention_rows_kernel<__half, true, 64>);
        return bf ? go(attention_rows_kernel<__nv_bfloat16, true, 128>) : go(attention_rows_kernel<__half, true, 128>);
    }
    if (D == 64) return bf ? go(attention_rows_kernel<__nv_bfloat16, false, 64>) : go(attention_rows_kernel<__half, false, 64>);
    return bf ? go(attention_rows_kernel<__nv_bfloat16, false, 128>) : go(attention_rows_kernel<__half, false, 128>);
}

}  // namespace hora
