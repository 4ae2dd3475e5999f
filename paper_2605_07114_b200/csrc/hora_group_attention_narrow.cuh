// hora_group_attention: narrow items, up to 8, 16 or 24 query rows: decode of single tokens over long caches.
//
// The call is bound by the cache's bytes (16 rows or fewer to a key: at most 16 products a byte), so the tensor unit matters only in
// that it has to be out of the way, and what counts is bytes in flight.  Every warp is a stream of its own, with its own
// running maximum, sum and output and its own ring of stages in shared memory: a stage is the keys and values of a step, fetched by
// cp.async (16 KiB of stages a warp, twelve warps an SM: up to 192 KiB in flight, several times what 6.5 TB/s needs at
// the latency of HBM under load).  No barrier joins the warps, and none waits for another.
//
// From the ring the operands go into the registers of mma.m16n8k16 by 16-byte loads, with no transposition.  Keys and values
// are its left operand (16 keys, or 16 dimensions), queries and weights the right one (8 query rows): a key has few query rows to it,
// and so none of them is padding up to eight.
//   - scores S^T = K Q^T sum over the head's dimensions, in any order that Q and K agree on: lane (n, c) = (lane / 4, lane % 4)
//     takes 16 neighbouring bytes of a key, and the four lanes of a key neighbouring blocks of 16;
//   - O^T += V^T P^T sums over keys, two to a register: lane (n, c) loads 16 bytes of the two keys from dimension n * 8 (16 for
//     one-byte values) on and pairs them up by byte permutations.  Row n of the j-th product is then dimension n * 8 + j of the
//     head: a lane ends up with runs of neighbouring dimensions, which it stores as they are.  The weights come out of the first
//     product as (key, row) and go into the second as (row, key): one movmatrix for eight keys.
// The 16-byte chunks of a row lie at places exchanged by the row's number, and index n stands for key key_of(n), such that the eight
// lanes of each phase of a load hit different banks, for keys and for values.
//
// An e4m3 cache is multiplied in fp16, which holds its codes exactly: a key row's power-of-two scale is applied to its score, and a value
// row's goes into the exponent of its weight, 2^(s + e_v - m_o).  m_o is a reference of its own beside m, raised like it when an
// exponent exceeds it by 2^8: the largest weight times scale among the keys a row sees is then near 1 however far apart the scales are, and
// what fp16 cannot hold is 2^-24 and less of that.  A value row of zeros has the scale 1, which says nothing about it: where m_o is
// to be raised, such rows are found in the stage and left out.  l stays relative to m, and o is brought to m when the partial is stored.
// Queries are scaled by a power of two to lie well within fp16's range.
//   Measured: 480 rollouts of 1024 keys on average, 4 cache heads of 128, bf16: 5.6 TB/s; 1920 of 768 keys, 2 cache heads of 128, e4m3: 175 us
// for 0.86 GB, half of the issue slots.
#pragma once

#include <type_traits>

#include "hora_group_attention.cuh"

namespace hora {

// Tiles of 128-byte rows are swizzled by address: they begin at multiples of 1024.
extern __shared__ __align__(1024) uint8_t s_attention[];

constexpr int kRingBytes = 16384;                        // stages of one warp

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

// over the eight lanes that hold the same two query rows
__device__ __forceinline__ float rows_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(kFull, v, 4));
    v = fmaxf(v, __shfl_xor_sync(kFull, v, 8));
    return fmaxf(v, __shfl_xor_sync(kFull, v, 16));
}
__device__ __forceinline__ float rows_sum(float v) {
    v += __shfl_xor_sync(kFull, v, 4);
    v += __shfl_xor_sync(kFull, v, 8);
    return v + __shfl_xor_sync(kFull, v, 16);
}
// an 8 x 8 matrix of 16-bit values over the warp, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
    uint32_t t;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(v));
    return t;
}

__device__ __forceinline__ float exponent_byte(uint32_t b) { return __uint_as_float(b ? b << 23 : 0x400000u); }

// Shared memory by address: 0 where an access of `bytes` bytes at `at` lies in the kernel's.
__device__ __forceinline__ uint32_t in_shared(uint32_t at, uint32_t bytes) {
    uint32_t size;
    asm("mov.u32 %0, %%dynamic_smem_size;" : "=r"(size));
    return at - (uint32_t)__cvta_generic_to_shared(s_attention) <= size - bytes ? 0u : 1u;
}

__device__ __forceinline__ void copy16(uint32_t to, const void *from) {
    if (!HORA_IN(in_shared(to, 16), 1)) return;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

__device__ __forceinline__ uint4 lds16(uint32_t at) {
    if (!HORA_IN(in_shared(at, 16), 1)) return make_uint4(0, 0, 0, 0);
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
    if (!HORA_IN(in_shared(at, 8), 1)) return make_uint2(0, 0);
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
__device__ __forceinline__ uint32_t lds1(uint32_t at) {
    if (!HORA_IN(in_shared(at, 1), 1)) return 0u;
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}

// A stage of a warp's ring: keys, values, and (one-byte types) their scale bytes.
template <bool F8, int D>
struct Stage {
    static constexpr int kRowBytes = F8 ? D : 2 * D;
    static constexpr int kKeys = narrow_keys(F8, D);
    static constexpr int kHalf = kKeys * kRowBytes;                           // keys; values follow
    static constexpr int kStages = kRingBytes / (2 * kHalf);
    static constexpr int kExpBytes = F8 ? 2 * kKeys : 0;
    static constexpr int kBytes = 2 * kHalf;
    static constexpr int kWarpBytes = kStages * (kBytes + kExpBytes);         // scale bytes of all stages behind the rows
    static constexpr int kChunks = kRowBytes / 16;

    // place of 16-byte chunk `chunk` of row `row`
    static __device__ __forceinline__ uint32_t place(int row, int chunk) {
        if constexpr (kRowBytes == 64) return (row >> 1) * 128 + ((((row & 1) * 4 + chunk) ^ (row & 6)) << 4);
        else return row * kRowBytes + ((chunk ^ (row & 7)) << 4);
    }
    // key that index n (below 8) of a product stands for
    static __device__ __forceinline__ int key_of(int n) { return kRowBytes == 64 ? n : n ^ ((n & 1) << 2); }
};

// One stream, by one warp, with its ring at `ring` in shared memory; items of NT * 8 rows.
template <typename Q, bool F8, int D, int NT>
__device__ __forceinline__ void narrow_stream(const AttnArgs &a, int32_t stream, uint32_t ring) {
    using M = std::conditional_t<F8, __half, Q>;                  // the type of the products
    using St = Stage<F8, D>;
    constexpr int kBlocks = F8 ? D / 64 : D / 32;                 // 16-byte loads of a lane for each key in K
    constexpr int kHalves = F8 ? 1 : D / 64;                      // and for each key in V (one-byte values, D = 64: 8 bytes)
    constexpr int kSteps = D / 16;                                // products over D for scores, tiles of 16 dimensions of the output
    constexpr int kRun = F8 ? D / 8 : 8;                          // neighbouring dimensions that a lane holds of the output
    constexpr int kRows = NT * 8;
    constexpr int kStages = St::kStages, kKeys = St::kKeys, kSixteens = kKeys / 16;
    const int lane = lane_id();
    const int n = lane >> 2, c = lane & 3;
    const uint32_t exps = ring + kStages * St::kBytes;
    const int64_t rows_all = (int64_t)a.R * a.T * a.Hq;
    bool bad = false;
    Pieces<false> pieces(a, stream, bad);
    Piece w;

    // where this lane reads: keys key_of(n), key_of(n) + 8 for the scores, and the two keys of indices 2c and 2c + 1 (and
    // those eight further on) for the product with the weights
    const int key_n = St::key_of(n), key_a = St::key_of(2 * c), key_b = St::key_of(2 * c + 1);

    while (pieces.next(a, w, bad)) {
        const Sequence &s = pieces.s;
        const int32_t step0 = w.step0, step1 = w.step1, h = w.h;

        // page numbers are looked up one step before the copies that need them
        struct Ids { int32_t id[kSixteens]; };
        auto pages_of = [&](int32_t step) {
            Ids p;
#pragma unroll
            for (int y = 0; y < kSixteens; ++y) {
                const int32_t key = step * kKeys + y * 16;
                p.id[y] = step < step1 && key < s.len && HORA_IN(key >> a.page_shift, w.prompt ? a.prefix_ld : a.suffix_ld) ? __ldcg(w.pages + (key >> a.page_shift)) : 0;
            }
            return p;
        };
        auto fetch = [&](int32_t step, const Ids &p) {
            if (step < step1) {
                const int slot = (step - step0) % kStages;
                const uint32_t to = ring + slot * St::kBytes;
#pragma unroll
                for (int y = 0; y < kSixteens; ++y) {             // sixteen keys lie in one page, one after the other
                    const int32_t key = step * kKeys + y * 16;
                    if (key >= s.len) break;
                    int32_t page = p.id[y];
                    if (page < 0 || page >= a.n_pages) { bad = true; page = 0; }
                    const int64_t row = (((int64_t)page * a.Hkv + h) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
                    if (!HORA_IN(row + 15, (a.n_pages * a.Hkv) << a.page_shift)) break;
                    const uint8_t *k = static_cast<const uint8_t *>(a.k_cache) + row * St::kRowBytes + lane * 16;
                    const uint8_t *v = static_cast<const uint8_t *>(a.v_cache) + row * St::kRowBytes + lane * 16;
#pragma unroll
                    for (int x = 0; x < St::kRowBytes / 32; ++x) {
                        const int chunk = x * kWarp + lane;
                        copy16(to + St::place(y * 16 + chunk / St::kChunks, chunk % St::kChunks), k + x * 512);
                    }
#pragma unroll
                    for (int x = 0; x < St::kRowBytes / 32; ++x) {
                        const int chunk = x * kWarp + lane;
                        copy16(to + St::kHalf + St::place(y * 16 + chunk / St::kChunks, chunk % St::kChunks), v + x * 512);
                    }
                    if (F8 && lane < 2) copy16(exps + slot * St::kExpBytes + lane * kKeys + y * 16, (lane == 0 ? a.k_exp : a.v_exp) + row);
                }
            }
            copies_done();                                        // a group for each step, empty ones too: the waits count groups
        };
        Ids page[kStages];
#pragma unroll
        for (int x = 0; x < kStages; ++x) page[x] = pages_of(step0 + x);
#pragma unroll
        for (int x = 0; x < kStages; ++x) fetch(step0 + x, page[x]);
        Ids page_next = pages_of(step0 + kStages);

        // queries: lane (n, c) has row n of each eight, in the dimensions that it takes of the keys
        uint32_t qf[NT][kSteps][2];
        float to_log2[NT][2];                                     // of rows 2c and 2c + 1, which are this lane's in the products
        int32_t limit[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const QueryRow row = query_row(a, s.first, s.rows, s.len, w.prompt, h, w.row0 + t * 8 + n);
            constexpr int kLoads = kBlocks * (F8 ? 2 : 1);
            const bool have = row.out >= 0 && HORA_IN(row.out, rows_all);
            const Q *from = static_cast<const Q *>(a.q) + (have ? row.out / a.Hq * a.q_row_stride + row.out % a.Hq * D : 0);
            uint4 x[kLoads];
#pragma unroll
            for (int b = 0; b < kLoads; ++b) {
                const int dim = F8 ? (b >> 1) * 64 + c * 16 + (b & 1) * 8 : b * 32 + c * 8;
                x[b] = have ? __ldcg(reinterpret_cast<const uint4 *>(from + dim)) : make_uint4(0, 0, 0, 0);
            }
            float unit = 1.f;                                     // what the stored queries have to be multiplied by
            if constexpr (F8) {
                // to fp16 with the row's largest value in [64, 128): smaller ones keep 11 bits down to 2^-21 of it
                float top = 0.f, y[kLoads][8];
#pragma unroll
                for (int b = 0; b < kLoads; ++b) {
                    widen8(Raw8<Q>{x[b]}, y[b]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(y[b][e]));
                }
                top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
                top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
                const int e2 = (int)(__float_as_uint(top) >> 23) - 127 - 6;
                if (top > 0.f && e2 < 120) unit = __uint_as_float((uint32_t)(max(e2, -120) + 127) << 23);
                const float f = 1.f / unit;                       // powers of two: exact
#pragma unroll
                for (int b = 0; b < kLoads; ++b) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[b][e] *= f;
                    x[b] = pack8<__half>(y[b]);
                }
            }
#pragma unroll
            for (int b = 0; b < kLoads; ++b) {
                qf[t][2 * b][0] = x[b].x;
                qf[t][2 * b][1] = x[b].y;
                qf[t][2 * b + 1][0] = x[b].z;
                qf[t][2 * b + 1][1] = x[b].w;
            }
            // row r's values lie in lanes 4r .. 4r + 3
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                to_log2[t][e] = a.scale_log2 * __shfl_sync(kFull, unit, (2 * c + e) * 4);
                limit[t][e] = __shfl_sync(kFull, row.limit, (2 * c + e) * 4);
            }
        }
        // keys that every query of the piece sees
        const int32_t open = w.prompt ? s.len : s.len - a.T + 1;

        float o[kSteps][NT][4] = {};
        float m[NT][2], l[NT][2], m_o[NT][2];                     // m_o: F8, what o is relative to
#pragma unroll
        for (int t = 0; t < NT; ++t) m[t][0] = m[t][1] = m_o[t][0] = m_o[t][1] = -INFINITY, l[t][0] = l[t][1] = 0.f;
        for (int32_t step = step0; step < step1; ++step) {
            const int32_t key = step * kKeys;
            const int slot = (step - step0) % kStages;
            const uint32_t at_k = ring + slot * St::kBytes, at_v = at_k + St::kHalf, at_ke = exps + slot * St::kExpBytes, at_ve = at_ke + kKeys;
            copies_wait<kStages - 1>();
            __syncwarp();
            float sc[kSixteens][NT][4];                           // keys key_n, key_n + 8 by rows 2c, 2c + 1
#pragma unroll
            for (int y = 0; y < kSixteens; ++y) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[y][t][e] = 0.f;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    const uint4 x0 = lds16(at_k + St::place(y * 16 + key_n, b * 4 + c)), x1 = lds16(at_k + St::place(y * 16 + 8 + key_n, b * 4 + c));
                    const uint32_t k0[4] = {x0.x, x0.y, x0.z, x0.w}, k1[4] = {x1.x, x1.y, x1.z, x1.w};
                    if constexpr (F8) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t kf[4] = {e4m3x2_to_half2(k0[e] & 0xFFFFu), e4m3x2_to_half2(k1[e] & 0xFFFFu), e4m3x2_to_half2(k0[e] >> 16), e4m3x2_to_half2(k1[e] >> 16)};
#pragma unroll
                            for (int t = 0; t < NT; ++t) mma16816(sc[y][t], kf, qf[t][4 * b + e][0], qf[t][4 * b + e][1], M());
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t kf[4] = {k0[2 * e], k1[2 * e], k0[2 * e + 1], k1[2 * e + 1]};
#pragma unroll
                            for (int t = 0; t < NT; ++t) mma16816(sc[y][t], kf, qf[t][2 * b + e][0], qf[t][2 * b + e][1], M());
                        }
                    }
                }
            }
            // scores in units of log2, hidden keys at -infinity
            float ve[kSixteens][2] = {};                          // F8: the exponents of the value scales
#pragma unroll
            for (int y = 0; y < kSixteens; ++y)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int k = y * 16 + x * 8 + key_n;
                    const float f = F8 ? exponent_byte(lds1(at_ke + k)) : 1.f;
                    // the byte behind the bits of 2^23 is 2^23 + byte; beyond the length it may be any, and the score is -infinity
                    if constexpr (F8) ve[y][x] = __uint_as_float(0x4B000000u | lds1(at_ve + k)) - (8388608.f + 127.f);
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 2; ++e) sc[y][t][2 * x + e] *= F8 ? to_log2[t][e] * f : to_log2[t][e];
                }
            if (key + kKeys > open) {
#pragma unroll
                for (int y = 0; y < kSixteens; ++y)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (key + y * 16 + (e >> 1) * 8 + key_n >= limit[t][e & 1]) sc[y][t][e] = -INFINITY;
            }
            // The reference of a row is raised when a score exceeds it by 2^8: weights up to 256 are as exact as weights up
            // to 1, and the output is hardly ever rescaled.
            bool raise = false;
            float top[NT][2];
            auto top_with_scale = [&](int t, int e) {             // F8: the largest s + e_v of this lane's keys
                float x = fmaxf(sc[0][t][e] + ve[0][0], sc[0][t][2 + e] + ve[0][1]);
#pragma unroll
                for (int y = 1; y < kSixteens; ++y) x = fmaxf(x, fmaxf(sc[y][t][e] + ve[y][0], sc[y][t][2 + e] + ve[y][1]));
                return x;
            };
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[t][e] = fmaxf(sc[0][t][e], sc[0][t][2 + e]);
#pragma unroll
                    for (int y = 1; y < kSixteens; ++y) top[t][e] = fmaxf(top[t][e], fmaxf(sc[y][t][e], sc[y][t][2 + e]));
                    raise |= top[t][e] > m[t][e] + 8.f;
                    if constexpr (F8) raise |= top_with_scale(t, e) > m_o[t][e] + 8.f;
                }
            if (__any_sync(kFull, raise)) {
                if constexpr (F8) {
                    // rows of zeros: a lane to each of the step's values (what was not fetched is any, and its score -infinity)
                    static_assert(kKeys == kWarp, "a lane to each key");
                    uint32_t bits = 0u;
#pragma unroll
                    for (int x = 0; x < St::kChunks; ++x) {
                        const uint4 v = lds16(at_v + St::place(lane, x));
                        bits |= v.x | v.y | v.z | v.w;
                    }
                    const unsigned zeros = __ballot_sync(kFull, (bits & 0x7F7F7F7Fu) == 0u);
#pragma unroll
                    for (int y = 0; y < kSixteens; ++y)
#pragma unroll
                        for (int x = 0; x < 2; ++x)
                            if (zeros >> (y * 16 + x * 8 + key_n) & 1u) ve[y][x] = -INFINITY;
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float up = fmaxf(m[t][e], rows_max(top[t][e])), f = up == -INFINITY ? 0.f : exp2_fast(m[t][e] - up);
                        m[t][e] = up;
                        l[t][e] *= f;
                        float f_o = f;
                        if constexpr (F8) {
                            const float up_o = fmaxf(m_o[t][e], rows_max(top_with_scale(t, e)));
                            f_o = up_o == -INFINITY ? 0.f : exp2_fast(m_o[t][e] - up_o);
                            m_o[t][e] = up_o;
                        }
#pragma unroll
                        for (int d = 0; d < kSteps; ++d) {
                            o[d][t][e] *= f_o;
                            o[d][t][2 + e] *= f_o;
                        }
                    }
            }
            uint32_t p[kSixteens][NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                // where no key has been seen the reference is -infinity and every weight has to come out as 0
                const float z0 = m[t][0] == -INFINITY ? 0.f : m[t][0], z1 = m[t][1] == -INFINITY ? 0.f : m[t][1];
                const float y0 = m_o[t][0] == -INFINITY ? 0.f : m_o[t][0], y1 = m_o[t][1] == -INFINITY ? 0.f : m_o[t][1];
#pragma unroll
                for (int y = 0; y < kSixteens; ++y)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float w0 = exp2_fast(sc[y][t][2 * x] - z0), w1 = exp2_fast(sc[y][t][2 * x + 1] - z1);
                        l[t][0] += w0;
                        l[t][1] += w1;
                        if constexpr (F8) {
                            w0 = exp2_fast(sc[y][t][2 * x] + ve[y][x] - y0);
                            w1 = exp2_fast(sc[y][t][2 * x + 1] + ve[y][x] - y1);
                        }
                        p[y][t][x] = transposed(pack2(w0, w1, M()));
                    }
            }
#pragma unroll
            for (int y = 0; y < kSixteens; ++y) {
                if (y > 0 && key + y * 16 >= s.len) break;        // those keys were not fetched
#pragma unroll
                for (int b = 0; b < kHalves; ++b) {
                    uint32_t v[4][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int k = y * 16 + (j >> 1) * 8 + ((j & 1) ? key_b : key_a);
                        uint4 x;
                        if constexpr (F8 && D == 64) {
                            const uint2 x2 = lds8(at_v + St::place(k, n >> 1) + (n & 1) * 8);
                            x = make_uint4(x2.x, x2.y, 0u, 0u);
                        } else {
                            x = lds16(at_v + St::place(k, b * 8 + n));
                        }
                        v[j][0] = x.x;
                        v[j][1] = x.y;
                        v[j][2] = x.z;
                        v[j][3] = x.w;
                    }
                    if (key + y * 16 + 16 > s.len) {              // what lies beyond the length may be anything, and 0 * NaN is not 0
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (key + y * 16 + (j >> 1) * 8 + ((j & 1) ? key_b : key_a) >= s.len) v[j][0] = v[j][1] = v[j][2] = v[j][3] = 0u;
                    }
                    if constexpr (F8) {
#pragma unroll
                        for (int q = 0; q < kSteps / 2; ++q) {    // four dimensions of a key to a word
                            const uint32_t lo0 = __byte_perm(v[0][q], v[1][q], 0x5140), hi0 = __byte_perm(v[0][q], v[1][q], 0x7362);
                            const uint32_t lo1 = __byte_perm(v[2][q], v[3][q], 0x5140), hi1 = __byte_perm(v[2][q], v[3][q], 0x7362);
                            const uint32_t vf0[4] = {e4m3x2_to_half2(lo0 & 0xFFFFu), e4m3x2_to_half2(lo0 >> 16), e4m3x2_to_half2(lo1 & 0xFFFFu), e4m3x2_to_half2(lo1 >> 16)};
                            const uint32_t vf1[4] = {e4m3x2_to_half2(hi0 & 0xFFFFu), e4m3x2_to_half2(hi0 >> 16), e4m3x2_to_half2(hi1 & 0xFFFFu), e4m3x2_to_half2(hi1 >> 16)};
#pragma unroll
                            for (int t = 0; t < NT; ++t) {
                                mma16816(o[2 * q][t], vf0, p[y][t][0], p[y][t][1], M());
                                mma16816(o[2 * q + 1][t], vf1, p[y][t][0], p[y][t][1], M());
                            }
                        }
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {             // two dimensions of a key to a word
                            const uint32_t vf[4] = {__byte_perm(v[0][q], v[1][q], 0x5410), __byte_perm(v[0][q], v[1][q], 0x7632),
                                                    __byte_perm(v[2][q], v[3][q], 0x5410), __byte_perm(v[2][q], v[3][q], 0x7632)};
#pragma unroll
                            for (int t = 0; t < NT; ++t) mma16816(o[4 * b + q][t], vf, p[y][t][0], p[y][t][1], M());
                        }
                    }
                }
            }
            __syncwarp();                                         // every lane has read the stage that is filled next
            fetch(step + kStages, page_next);
            page_next = pages_of(step + kStages + 1);
        }

        // o[d][t] holds rows 2c, 2c + 1 of the t-th eight, each in dimensions n * kRun + 2d and the next one (by parts of 8 * kRun)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float sum = rows_sum(l[t][e]);
                // F8: o from m_o to m, in two steps, since 2^(m_o - m) by itself can pass fp32's range
                if constexpr (F8) {
                    const float f = m_o[t][e] == -INFINITY ? 0.f : exp2_fast(0.5f * (m_o[t][e] - m[t][e]));
#pragma unroll
                    for (int d = 0; d < kSteps; ++d) {
                        o[d][t][e] = o[d][t][e] * f * f;
                        o[d][t][2 + e] = o[d][t][2 + e] * f * f;
                    }
                }
                const int32_t x = t * 8 + 2 * c + e;
                const int64_t out = query_row(a, s.first, s.rows, s.len, w.prompt, h, w.row0 + x).out;
                if (out < 0) continue;
                const int64_t place = step0 > 0 ? (int64_t)stream * kRows + x : (w.prompt ? kPromptPart : kOwnPart) * rows_all + out;
                if (!HORA_IN(place, step0 > 0 ? (int64_t)a.n_narrow * kRows : 2 * rows_all)) continue;
                float *po = (step0 > 0 ? a.cont_o[0] : a.main_o) + place * D;
#pragma unroll
                for (int part = 0; part < D / (8 * kRun); ++part)
#pragma unroll
                    for (int d = 0; d < kRun / 2; d += 2)
                        *reinterpret_cast<float4 *>(po + part * 8 * kRun + n * kRun + 2 * d) =
                            make_float4(o[part * (kRun / 2) + d][t][e], o[part * (kRun / 2) + d][t][2 + e], o[part * (kRun / 2) + d + 1][t][e],
                                        o[part * (kRun / 2) + d + 1][t][2 + e]);
                if (n == 0) *reinterpret_cast<float2 *>((step0 > 0 ? a.cont_ml[0] : a.main_ml) + place * 2) = make_float2(m[t][e], sum);
            }
    }
    if (bad) raise_status(a.status, HORA_ERR_INVALID_VALUE);
}

}  // namespace hora
