// hora_packed_attention_backward: gradients of keys and values, and of queries.
//
//   P = 2^(scale q.k - lse) (in units of log2),  dP = dout . v,  dS = P (dP - dout . out)
//   dV = P^T dO, dK = scale dS^T Q  (sums over queries and the heads of a cache head)      dQ = scale dS K  (a sum over keys)
//
// Two kernels, each with its sums in tensor memory from the first step to the last, so no sum depends on an order and nothing is
// added up in memory; the price is that S and dP are computed twice (seven products where five would do).
//   Keys: an item is 128 keys of one cache head and all queries that may see them, 128 rows (tokens times heads) a step.  S^T = K Q^T and dP^T = V dO^T
// have the keys as rows: P^T and dS^T replace them in tensor memory in 16 bits and are the left operands of dV += P^T dO and dK += dS^T Q, for
// which the same tiles of dO and Q are read the other way round.  Nothing but the four operands ever is in shared memory.
//   Queries: an item is one tile of queries; S = Q K^T, dP = dO V^T, dQ += dS K.  Here dS enters its product twice, as its value in 16 bits and as
// what that rounding left: dQ is then off by the roundings of the result and of dout . out alone.  A row's dS add up to nothing; what they do add up
// to is what dout . out of the rounded output was off by, so this kernel runs first and leaves it for the keys' one.  (Relative error of dq,
// dk in bf16 2.3e-3 in place of 2.6e-3 to 2.9e-3; 1327 us in place of 1140 for 128 rollouts up to 1021 tokens in 8 groups, 28 heads of 128.)
//   Eight warps do what is between the products, two threads to a row, 64 columns each.  Keys: the products come in the order dV, next S^T, dK, next dP^T,
// so that the weights of a step wait for its S^T alone.  Queries: dP is a step ahead in two places.
//   What bounds them: the keys' kernel, the chain of a step (3.7 thousand cycles, of which the products take 2.05: 1.5 ms for those rollouts, 0.64 ms
// for two traces of 8191 tokens and 16 heads, 1.0 PFLOP/s); the queries' kernel, its products on long traces (68 % of the cycles).
//   Rows of a tile that are not of the run of queries (or keys) are cleared in shared memory where a product sums over them.
//   Every wait has a limit; a wait that reaches it makes the CTA give up and report HORA_ERR_INTERNAL.
#define HORA_FILE_ID 12
#include <type_traits>

#include "hora_packed_attention.cuh"

HORA_CHECKED_REGISTER()

namespace hora {

namespace {

constexpr int kTile = kPackedRows, kHalfTile = kTile / 2;
constexpr int kRest = kHalfTile / 2;                     // columns from gradients of scores to what rounding them left
constexpr int kMiddleThreads = 256, kLoadWarp = 8, kProductWarp = 9, kFeedWarp = 11;
constexpr int kFeedReaders = 11;                         // warps that take items from the feeder (one less for keys)

template <typename Q>
constexpr uint32_t kType = std::is_same<Q, __nv_bfloat16>::value ? 1u : 0u;
template <typename Q>
constexpr uint32_t kIdescScores = (1u << 4) | (kType<Q> << 7) | (kType<Q> << 10) | ((kTile / 16) << 24);                // and the columns / 8 at bit 17
template <typename Q, int D>
constexpr uint32_t kIdescSum = (1u << 4) | (kType<Q> << 7) | (kType<Q> << 10) | (1u << 16) | ((D / 8) << 17) | ((kTile / 16) << 24);

// The product over D of a tile's 128 rows `a` and the first `count` rows of `b` (up to a multiple of sixteen).  Whole warps, here and below.
template <typename Q, int D>
__device__ __forceinline__ void product_of_rows(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, int32_t count) {
    const uint32_t idesc = kIdescScores<Q> | (uint32_t)((count + 15) >> 4) << 18;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
        const uint32_t off = ((x >> 2) * (kTile * 128) + (x & 3) * 32) >> 4;
        mma_smem(lead, d, a + off, b + off, idesc, x > 0);
    }
}
// d += w b, w 128 x `count` in tensor memory (16 bits, its two halves of 64 columns 64 columns of 32 bits apart), b `count` rows of D.
template <typename Q, int D>
__device__ __forceinline__ void product_with_weights(uint32_t lead, uint32_t d, uint32_t w, uint32_t b, int32_t count, bool first) {
    mma_tmem(lead, d, w, b, kIdescSum<Q, D>, !first);
    if (count > kTile - 16) {
#pragma unroll
        for (int g = 1; g < kTile / 16; ++g) mma_tmem(lead, d, w + (g < 4 ? g * 8 : kHalfTile + (g - 4) * 8), b + g * (2048 >> 4), kIdescSum<Q, D>, 1);
    } else {
#pragma unroll 1
        for (int g = 1; g * 16 < count; ++g) mma_tmem(lead, d, w + g * 8 + (g < 4 ? 0 : kHalfTile - 32), b + g * (2048 >> 4), kIdescSum<Q, D>, 1);
    }
}

__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) { return half2_bits(w); }

// Rows count .. of a tile up to the last sixteen that a product reads are set to zero.  All lanes of a warp.
template <int D>
__device__ __forceinline__ void clear_rows(uint32_t tile, int32_t count) {
    const int32_t clear = ((count + 15) & ~15) - count;
    for (int32_t c = lane_id(); c < clear * (D / 8); c += kWarp) {
        const uint32_t to = tile + (c % (D / 8) >> 3) * (kTile * 128) + (count + c / (D / 8)) * 128 + (c & 7) * 16;
        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(to), "r"(0) : "memory");
    }
}

__device__ __forceinline__ void publish_clears() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

template <int COLUMNS, typename Q>
__device__ __forceinline__ void store_row(Q *to, uint32_t from, float f, bool have) {
#pragma unroll 1
    for (int b = 0; b < COLUMNS / 32; ++b) {
        float o[32];
        tmem_load(from + b * 32, o);
        tmem_load_wait();
        if (have) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = o[v * 8 + e] * f;
                *reinterpret_cast<uint4 *>(to + b * 32 + v * 8) = pack8<Q>(x);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------
// keys and values

template <int D>
struct KeysSmem {
    static constexpr int kTileBytes = kTile * D * 2;
    static constexpr int kStages = D == 128 ? 2 : 4;
    static constexpr int kK = 0, kV = kTileBytes, kRing = 2 * kTileBytes;            // a stage: queries, gradients of outputs
    static constexpr int kSmall = kRing + kStages * 2 * kTileBytes;
};

struct KeysShared {
    Feed feed;
    float lse[4][kTile], delta[4][kTile];                // by stage: -lse, -dout.out, as the exponents and sums need them
    uint64_t full[4], empty[4], keys, keys_free, scores, weights, products, gradients, sums, sums_free;
    int32_t failed;
    uint32_t tmem;
};

struct KeyWork {
    int32_t key0, keys, q0, q1, head, steps, slot0, parts, part, ticket;
    bool valid;
};

__device__ __forceinline__ KeyWork make_keys(const PackedArgs &a, const FeedSlot &f) {
    KeyWork w;
    w.valid = f.valid;
    w.head = f.part;
    w.key0 = f.a.x;
    w.keys = f.a.y;
    w.q0 = f.a.z;
    w.q1 = f.a.w;
    w.slot0 = f.b.x;
    w.parts = f.b.y;
    w.part = f.b.z;
    w.ticket = f.b.w;
    w.steps = (f.a.w - f.a.z + a.tp - 1) / a.tp * (a.g / a.hp);
    return w;
}

// Step s: which tokens, which block of heads, how many rows.
struct KeyStep {
    int32_t token0, block, count;
    bool whole;
};
__device__ __forceinline__ KeyStep key_step(const PackedArgs &a, const KeyWork &w, int32_t s) {
    const int32_t per = a.g / a.hp, tile = s / per;
    KeyStep k;
    k.token0 = w.q0 + tile * a.tp;
    k.block = w.head * per + (s - tile * per);
    const int32_t tokens = min(a.tp, w.q1 - k.token0);
    k.count = tokens * a.hp;
    k.whole = tokens == a.tp;
    return k;
}

extern __shared__ __align__(1024) uint8_t s_backward[];

template <typename Q, int D>
__global__ void __launch_bounds__(kPackedThreads, 1)
packed_keys_kernel(const PackedArgs a, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap do_map,
                   const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    using Smem = KeysSmem<D>;
    constexpr uint32_t kStages = Smem::kStages;
    constexpr int kParts = D / 64;
    KeysShared &sh = *reinterpret_cast<KeysShared *>(s_backward + Smem::kSmall);
    const uint32_t base = smem_at(s_backward);
    const int warp = threadIdx.x >> 5, lane = lane_id();
    volatile int32_t *failed = &sh.failed;
    if (base & 1023u) {
        pdl_enter();
        raise_status(a.status, HORA_ERR_INTERNAL);
        return;
    }
    const uint32_t full = smem_at(sh.full), empty = smem_at(sh.empty), keys = smem_at(&sh.keys), keys_free = smem_at(&sh.keys_free), scores = smem_at(&sh.scores),
                   weights = smem_at(&sh.weights), products = smem_at(&sh.products), gradients = smem_at(&sh.gradients), sums = smem_at(&sh.sums),
                   sums_free = smem_at(&sh.sums_free);
    if (threadIdx.x == 0) {
        sh.failed = 0;
        feed_init(sh.feed, kFeedReaders - 1);
        for (uint32_t s = 0; s < kStages; ++s) {
            bar_init(full + 8 * s, 1 + kWarp);
            bar_init(empty + 8 * s, 1);
        }
        bar_init(keys, 1);
        bar_init(keys_free, 1);
        bar_init(scores, 1);
        bar_init(weights, kMiddleThreads);
        bar_init(products, 1);
        bar_init(gradients, kMiddleThreads);
        bar_init(sums, 1);
        bar_init(sums_free, kMiddleThreads);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // rows that no tile of queries fills
    const int32_t rows = a.hp * a.tp, idle = kTile - rows;
    for (int32_t c = threadIdx.x; c < 2 * (int32_t)kStages * kParts * idle * 8; c += kPackedThreads) {
        const int32_t x = c >> 3, part = x / idle;
        const uint32_t to = base + Smem::kRing + part * (kTile * 128) + (rows + x - part * idle) * 128 + (c & 7) * 16;
        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(to), "r"(0) : "memory");
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_at(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = sh.tmem;                       // columns: S^T, dP^T, dV, dK
    pdl_enter();
    const int shift = gradient_shift(a), up = a.half ? kHalfShift : 0;
    bool ok = true;

    if (warp == kFeedWarp) {
        if (lane == 0) feed<2>(sh.feed, reinterpret_cast<const int4 *>(a.key_items), __ldcg(a.counts + 1), a.key_cap, a.Hkv, a.counts + 5, failed);
    } else if (warp == kLoadWarp) {
        // ---- keys, values, tiles of queries and of gradients of outputs; and of each row of a step -lse and -dout.out
        const float c = exp2f((float)(shift - up));
        uint32_t pos = 0, r = 0;
        for (; ok; ++r) {
            const KeyWork it = make_keys(a, feed_next<false>(sh.feed, r, failed));
            if (!it.valid) break;
            if (r > 0) ok = __all_sync(kFull, bar_wait(keys_free, (r + 1) & 1, failed));
            if (!ok) break;
            if (lane == 0) {
                bar_expect(keys, 2 * Smem::kTileBytes);
                for (int p = 0; p < kParts; ++p) {
                    tma_box3(base + Smem::kK + p * (kTile * 128), &k_map, p * 64, it.head, it.key0, keys);
                    tma_box3(base + Smem::kV + p * (kTile * 128), &v_map, p * 64, it.head, it.key0, keys);
                }
            }
            __syncwarp();
            auto stats_of = [&](int32_t s, float4 (&st)[kTile / kWarp]) {
                const KeyStep k = key_step(a, it, s);
#pragma unroll
                for (int i = 0; i < kTile / kWarp; ++i) {
                    const int32_t row = lane + i * kWarp, token = k.token0 + row / a.hp;
                    st[i] = make_float4(INFINITY, 0.f, 0.f, 0.f);
                    if (row < k.count && HORA_IN(token, a.T)) st[i] = __ldcg(a.stats + (int64_t)token * a.Hq + k.block * a.hp + row % a.hp);
                }
            };
            float4 st[kTile / kWarp];
            stats_of(0, st);
            for (int32_t s = 0; s < it.steps; ++s, ++pos) {
                const KeyStep k = key_step(a, it, s);
                const uint32_t stage = pos % kStages;
                if (pos >= kStages) ok = __all_sync(kFull, bar_wait(empty + 8 * stage, (pos / kStages + 1) & 1, failed));
                if (!ok) break;
                if (lane == 0) {
                    bar_expect(full + 8 * stage, 2 * kParts * rows * 128);
                    const uint32_t at = base + Smem::kRing + stage * 2 * Smem::kTileBytes;
                    for (int p = 0; p < kParts; ++p) {
                        tma_box3(at + p * (kTile * 128), &q_map, p * 64, k.block * a.hp, k.token0, full + 8 * stage);
                        tma_box3(at + Smem::kTileBytes + p * (kTile * 128), &do_map, p * 64, k.block * a.hp, k.token0, full + 8 * stage);
                    }
                }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < kTile / kWarp; ++i) {
                    sh.lse[stage][lane + i * kWarp] = (float)up - st[i].x;
                    sh.delta[stage][lane + i * kWarp] = -(st[i].y + (st[i].z + st[i].w)) * c;
                }
                bar_arrive(full + 8 * stage);
                if (s + 1 < it.steps) stats_of(s + 1, st);
            }
        }
        if (*failed && lane == 0) {                      // copies on their way to the CTA
            int32_t never = 0;
            if (r > 0) bar_wait(keys, (r - 1) & 1, &never);
            for (uint32_t x = pos < kStages ? 0 : pos - kStages; x < pos; ++x) bar_wait(full + 8 * (x % kStages), (x / kStages) & 1, &never);
        }
    } else if (warp == kProductWarp) {
        // ---- products, in the order dV, the next S^T, dK, the next dP^T: the weights of a step wait for its S^T alone, while dK and dP^T are under way.
        // A wait that has failed is not looked at here: what follows is of no use, but in bounds, and there is no next item
        const uint32_t lead = elect_one(), k_rows = operand(base + Smem::kK, 16), v_rows = operand(base + Smem::kV, 16);
        uint32_t phase = 0, pos = 0;
        for (uint32_t r = 0;; ++r) {
            const KeyWork it = make_keys(a, feed_next<false>(sh.feed, r, failed));
            if (!it.valid) break;
            int32_t count = 0;
            auto tile = [&](uint32_t x, int which, uint32_t lead_bytes) {
                return operand(base + Smem::kRing + (x % kStages * 2 + which) * Smem::kTileBytes, lead_bytes);
            };
            bar_wait(keys, r & 1, failed);
#pragma unroll 1
            for (int32_t s = -1; s < it.steps; ++s, ++pos) {                 // pos: the place of step s + 1
                if (s >= 0) {
                    bar_wait(weights, phase, failed);
                    if (s == 0 && r > 0) bar_wait(sums_free, (r + 1) & 1, failed);
                    fence_after();
                    product_with_weights<Q, D>(lead, tmem + 256, tmem, tile(pos - 1, 1, kTile * 128), count, s == 0);
                }
                int32_t next_count = 0;
                const bool more = s + 1 < it.steps;
                if (more) {
                    bar_wait(full + 8 * (pos % kStages), pos / kStages & 1, failed);
                    const KeyStep k = key_step(a, it, s + 1);
                    next_count = k.count;
                    if (!k.whole && (k.count & 15)) {    // rows of others
                        const uint32_t at = base + Smem::kRing + pos % kStages * 2 * Smem::kTileBytes;
                        clear_rows<D>(at, k.count);
                        clear_rows<D>(at + Smem::kTileBytes, k.count);
                        publish_clears();
                    }
                    fence_after();
                    product_of_rows<Q, D>(lead, tmem, k_rows, tile(pos, 0, 16), next_count);
                    mma_commit(lead, scores);
                }
                if (s >= 0) {
                    bar_wait(gradients, phase, failed);
                    phase ^= 1;
                    fence_after();
                    product_with_weights<Q, D>(lead, tmem + 256 + D, tmem + kTile, tile(pos - 1, 0, kTile * 128), count, s == 0);
                    mma_commit(lead, empty + 8 * ((pos - 1) % kStages));
                }
                if (more) {
                    product_of_rows<Q, D>(lead, tmem + kTile, v_rows, tile(pos, 1, 16), next_count);
                    mma_commit(lead, products);
                }
                count = next_count;
            }
            --pos;
            mma_commit(lead, keys_free);
            mma_commit(lead, sums);
        }
    } else if (warp < 8) {
        // ---- between the products: thread `row` of either half has 64 columns (queries) of a key
        const int half = warp >> 2, row = threadIdx.x & (kTile - 1);
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
        const uint32_t t_s = lanes + half * kHalfTile, t_dp = lanes + kTile + half * kHalfTile;
        const float c = exp2f((float)(shift - up));
        const float2 scale2 = make_float2(a.scale_log2, a.scale_log2), c2 = make_float2(c, c);
        uint32_t phase = 0, pos = 0;
        for (int32_t r = 0; ok; ++r) {
            const KeyWork it = make_keys(a, feed_next<false>(sh.feed, r, failed));
            if (!it.valid) break;
            for (int32_t s = 0; s < it.steps; ++s, ++pos, phase ^= 1) {
                const KeyStep k = key_step(a, it, s);
                const uint32_t stage = pos % kStages;
                ok = bar_wait(full + 8 * stage, (pos / kStages) & 1, failed) && bar_wait(scores, phase, failed);
                ok = __all_sync(kFull, ok);
                if (!ok) break;
                fence_after();
                float p[2][32];
#pragma unroll
                for (int b = 0; b < 2; ++b) tmem_load(t_s + b * 32, p[b]);
                tmem_load_wait();
                const float4 *lse = reinterpret_cast<const float4 *>(sh.lse[stage] + half * kHalfTile);
                // causal: the query's token may not be in front of the key
                const bool border = a.causal && k.token0 < it.key0 + it.keys - 1;
                const int32_t from = border ? (it.key0 + row - k.token0) * a.hp - half * kHalfTile : 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float4 z = lse[b * 4 + e];
                        float *x = p[b >> 1] + (b & 1) * 16 + 4 * e;
                        float2 y0 = fma2(make_float2(x[0], x[1]), scale2, make_float2(z.x, z.y)), y1 = fma2(make_float2(x[2], x[3]), scale2, make_float2(z.z, z.w));
                        x[0] = exp2_approx(y0.x);
                        x[1] = exp2_approx(y0.y);
                        x[2] = exp2_approx(y1.x);
                        x[3] = exp2_approx(y1.y);
                        if (border) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (b * 16 + 4 * e + i < from) x[i] = 0.f;
                        }
                        w[2 * e] = pack2(x[0], x[1], Q());
                        w[2 * e + 1] = pack2(x[2], x[3], Q());
                    }
                    tmem_store8(t_s + b * 8, w);
                }
                tmem_store_wait();
                fence_before();
                bar_arrive(weights);
                ok = bar_wait(products, phase, failed);
                ok = __all_sync(kFull, ok);
                if (!ok) break;
                fence_after();
                const float4 *delta = reinterpret_cast<const float4 *>(sh.delta[stage] + half * kHalfTile);
                float dp[2][32];
#pragma unroll
                for (int b = 0; b < 2; ++b) tmem_load(t_dp + b * 32, dp[b]);
                tmem_load_wait();
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float4 z = delta[b * 4 + e];
                        const float *x = p[b >> 1] + (b & 1) * 16 + 4 * e, *d = dp[b >> 1] + (b & 1) * 16 + 4 * e;
                        const float2 y0 = mul2(make_float2(x[0], x[1]), fma2(make_float2(d[0], d[1]), c2, make_float2(z.x, z.y)));
                        const float2 y1 = mul2(make_float2(x[2], x[3]), fma2(make_float2(d[2], d[3]), c2, make_float2(z.z, z.w)));
                        w[2 * e] = pack2(y0.x, y0.y, Q());
                        w[2 * e + 1] = pack2(y1.x, y1.y, Q());
                    }
                    tmem_store8(t_dp + b * 8, w);
                }
                tmem_store_wait();
                fence_before();
                bar_arrive(gradients);
            }
            if (!ok) break;
            ok = bar_wait(sums, r & 1, failed);
            ok = __all_sync(kFull, ok);
            if (!ok) break;
            fence_after();
            Q *to = static_cast<Q *>(half ? a.dk : a.dv) + (int64_t)(it.key0 + row) * (half ? a.dk_stride : a.dv_stride) + (int64_t)it.head * D;
            const float factor = half ? a.scale * exp2f((float)-shift) : exp2f((float)-up);
            if (it.parts == 1) {
                store_row<D>(to, lanes + 256 + half * D, factor, row < it.keys && HORA_IN(it.key0 + row, a.T));
                fence_before();
                bar_arrive(sums_free);
            } else {
                // [slot][dV, dK][D / 4][128] of four values: neighbouring threads next to each other
                const int64_t slot = ((int64_t)it.slot0 * a.Hkv + it.head) * 2 + half, step = (int64_t)a.Hkv * 2;
                float4 *mine = reinterpret_cast<float4 *>(a.slots) + (slot + it.part * step) * (D / 4 * kTile) + row;
                if (HORA_IN(slot + it.part * step, 4 * a.n_sm)) {
#pragma unroll 1
                    for (int b = 0; b < D / 32; ++b) {
                        float o[32];
                        tmem_load(lanes + 256 + half * D + b * 32, o);
                        tmem_load_wait();
#pragma unroll
                        for (int v = 0; v < 8; ++v) mine[(b * 8 + v) * kTile] = make_float4(o[4 * v], o[4 * v + 1], o[4 * v + 2], o[4 * v + 3]);
                    }
                }
                fence_before();
                bar_arrive(sums_free);
                __threadfence();
                __syncwarp();
                const int32_t ticket = (it.ticket * a.Hkv + it.head) * 8 + warp;             // of the warp's rows
                int32_t before = 0;
                if (lane == 0 && HORA_IN(ticket, 8 * a.n_sm)) before = atomicAdd(a.tickets + ticket, 1);
                if (__shfl_sync(kFull, before, 0) == it.parts - 1) {     // the other parts are there: all of them, in their order
                    __threadfence();
                    const float4 *from = reinterpret_cast<const float4 *>(a.slots) + slot * (D / 4 * kTile) + row;
#pragma unroll 1
                    for (int b = 0; b < D / 16; ++b) {
                        float4 sum[4] = {};
                        for (int32_t x = 0; x < it.parts; x += 4) {          // sixteen loads in flight
                            float4 y[4][4];
#pragma unroll
                            for (int u = 0; u < 4; ++u)
#pragma unroll
                                for (int v = 0; v < 4; ++v)
                                    y[u][v] = x + u < it.parts ? __ldcg(from + (x + u) * step * (D / 4 * kTile) + (b * 4 + v) * kTile) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                            for (int u = 0; u < 4; ++u)
#pragma unroll
                                for (int v = 0; v < 4; ++v) {
                                    sum[v].x += y[u][v].x;
                                    sum[v].y += y[u][v].y;
                                    sum[v].z += y[u][v].z;
                                    sum[v].w += y[u][v].w;
                                }
                        }
                        if (row < it.keys && HORA_IN(it.key0 + row, a.T)) {
#pragma unroll
                            for (int v = 0; v < 4; v += 2) {
                                const float x[8] = {sum[v].x * factor, sum[v].y * factor, sum[v].z * factor, sum[v].w * factor,
                                                    sum[v + 1].x * factor, sum[v + 1].y * factor, sum[v + 1].z * factor, sum[v + 1].w * factor};
                                *reinterpret_cast<uint4 *>(to + b * 16 + v * 4) = pack8<Q>(x);
                            }
                        }
                    }
                }
            }
        }
    }
    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && sh.failed) raise_status(a.status, HORA_ERR_INTERNAL);
    if (warp == 0) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// ---------------------------------------------------------------------------------------------------------------
// queries

template <int D>
struct QueriesSmem {
    static constexpr int kTileBytes = kTile * D * 2;
    static constexpr int kKeyStages = D == 128 ? 3 : 4, kValueStages = D == 128 ? 2 : 4;
    static constexpr int kQ = 0, kDo = kTileBytes, kKeys = 2 * kTileBytes, kValues = kKeys + kKeyStages * kTileBytes, kSmall = kValues + kValueStages * kTileBytes;
};

struct QueriesShared {
    Feed feed;
    uint64_t full[8], empty[8], queries, queries_free, scores, scores_free, products[2], gradients[2], sums, sums_free;       // full, empty: keys, then values
    int32_t failed;
    uint32_t tmem;
};

struct QueryWork {
    int32_t token0, tokens, own0, end, shared0, shared1, block, n_shared, n, last;       // last: behind the last key that is seen of the own sequence
    bool valid;

    __device__ __forceinline__ int32_t key0(int32_t j) const { return j < n_shared ? shared0 + j * kTile : own0 + (j - n_shared) * kTile; }
    __device__ __forceinline__ int32_t count(int32_t j) const { return min(kTile, (j < n_shared ? shared1 : end) - key0(j)); }
    __device__ __forceinline__ int32_t seen(int32_t j) const { return min(kTile, (j < n_shared ? shared1 : last) - key0(j)); }
};

__device__ __forceinline__ QueryWork make_queries(const PackedArgs &a, const FeedSlot &f) {
    QueryWork w;
    w.valid = f.valid;
    w.block = f.part;
    w.token0 = f.a.x;
    w.tokens = f.a.y;
    w.own0 = f.a.z;
    w.end = f.a.w;
    w.shared0 = f.b.x;
    w.shared1 = f.b.y;
    w.n_shared = (f.b.y - f.b.x + kTile - 1) / kTile;
    w.last = a.causal ? f.a.x + f.a.y : f.a.w;
    w.n = w.n_shared + (w.last - f.a.z + kTile - 1) / kTile;
    return w;
}

template <typename Q, int D>
__global__ void __launch_bounds__(kPackedThreads, 1)
packed_queries_kernel(const PackedArgs a, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap do_map,
                      const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    using Smem = QueriesSmem<D>;
    constexpr uint32_t kKeyStages = Smem::kKeyStages, kValueStages = Smem::kValueStages;
    constexpr int kParts = D / 64;
    QueriesShared &sh = *reinterpret_cast<QueriesShared *>(s_backward + Smem::kSmall);
    const uint32_t base = smem_at(s_backward);
    const int warp = threadIdx.x >> 5, lane = lane_id();
    volatile int32_t *failed = &sh.failed;
    if (base & 1023u) {
        pdl_enter();
        raise_status(a.status, HORA_ERR_INTERNAL);
        return;
    }
    const uint32_t full = smem_at(sh.full), empty = smem_at(sh.empty), queries = smem_at(&sh.queries), queries_free = smem_at(&sh.queries_free),
                   scores = smem_at(&sh.scores), scores_free = smem_at(&sh.scores_free), products = smem_at(sh.products), gradients = smem_at(sh.gradients),
                   sums = smem_at(&sh.sums), sums_free = smem_at(&sh.sums_free);
    if (threadIdx.x == 0) {
        sh.failed = 0;
        feed_init(sh.feed, kFeedReaders);
        for (uint32_t s = 0; s < kKeyStages + kValueStages; ++s) {
            bar_init(full + 8 * s, 1);
            bar_init(empty + 8 * s, s < kKeyStages ? 2 : 1);             // both products' warps read keys
        }
        bar_init(queries, 1);
        bar_init(queries_free, 2);
        bar_init(scores, 1);
        bar_init(scores_free, kMiddleThreads);
        for (int b = 0; b < 2; ++b) {
            bar_init(products + 8 * b, 1);
            bar_init(gradients + 8 * b, kMiddleThreads);
        }
        bar_init(sums, 1);
        bar_init(sums_free, kMiddleThreads);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_at(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = sh.tmem;                       // columns: S, dP in two places, dQ
    pdl_enter();
    const int shift = gradient_shift(a), up = a.half ? kHalfShift : 0;
    bool ok = true;

    if (warp == kFeedWarp) {
        if (lane == 0) feed<2>(sh.feed, reinterpret_cast<const int4 *>(a.query_items), __ldcg(a.counts), a.query_cap, a.blocks, a.counts + 4, failed);
    } else if (warp == kLoadWarp) {
        if (lane == 0) {
            uint32_t pos = 0, r = 0;                     // steps so far
            auto bring = [&](uint32_t first, uint32_t stages, uint32_t to, const CUtensorMap *map, int32_t head, int32_t key0) {
                const uint32_t stage = pos % stages, bar = first + stage;
                if (pos >= stages) ok = bar_wait(empty + 8 * bar, (pos / stages + 1) & 1, failed);
                if (!ok) return;
                bar_expect(full + 8 * bar, Smem::kTileBytes);
                for (int p = 0; p < kParts; ++p) tma_box3(base + to + stage * Smem::kTileBytes + p * (kTile * 128), map, p * 64, head, key0, full + 8 * bar);
            };
            for (; ok; ++r) {
                const QueryWork it = make_queries(a, feed_next<true>(sh.feed, r, failed));
                if (!it.valid) break;
                const int32_t head = it.block * a.hp / a.g;
                if (r > 0) ok = bar_wait(queries_free, (r + 1) & 1, failed);
                if (!ok) break;
                bar_expect(queries, 2 * kParts * a.hp * a.tp * 128);
                for (int p = 0; p < kParts; ++p) {
                    tma_box3(base + Smem::kQ + p * (kTile * 128), &q_map, p * 64, it.block * a.hp, it.token0, queries);
                    tma_box3(base + Smem::kDo + p * (kTile * 128), &do_map, p * 64, it.block * a.hp, it.token0, queries);
                }
                for (int32_t j = 0; j < it.n && ok; ++j, ++pos) {
                    bring(0, kKeyStages, Smem::kKeys, &k_map, head, it.key0(j));
                    if (ok) bring(kKeyStages, kValueStages, Smem::kValues, &v_map, head, it.key0(j));
                }
            }
            if (*failed) {
                int32_t never = 0;
                if (r > 0) bar_wait(queries, (r - 1) & 1, &never);
                for (uint32_t x = pos < kKeyStages ? 0 : pos - kKeyStages; x < pos; ++x) bar_wait(full + 8 * (x % kKeyStages), x / kKeyStages & 1, &never);
                for (uint32_t x = pos < kValueStages ? 0 : pos - kValueStages; x < pos; ++x) bar_wait(full + 8 * (kKeyStages + x % kValueStages), x / kValueStages & 1, &never);
            }
        }
    } else if (warp == kProductWarp) {
        // ---- S.  As above, failed waits are not looked at by the warps with the products
        const uint32_t lead = elect_one(), q_rows = operand(base + Smem::kQ, 16);
        uint32_t pos = 0;
        for (uint32_t r = 0;; ++r) {
            const QueryWork it = make_queries(a, feed_next<false>(sh.feed, r, failed));
            if (!it.valid) break;
            bar_wait(queries, r & 1, failed);
#pragma unroll 1
            for (int32_t j = 0; j < it.n; ++j, ++pos) {
                const uint32_t stage = pos % kKeyStages;
                bar_wait(full + 8 * stage, pos / kKeyStages & 1, failed);
                if (pos > 0) bar_wait(scores_free, (pos + 1) & 1, failed);
                fence_after();
                product_of_rows<Q, D>(lead, tmem, q_rows, operand(base + Smem::kKeys + stage * Smem::kTileBytes, 16), it.seen(j));
                mma_commit(lead, scores);
                mma_commit(lead, empty + 8 * stage);
            }
            mma_commit(lead, queries_free);
        }
    } else if (warp == kProductWarp + 1) {
        // ---- dP, a step ahead, and dQ
        const uint32_t lead = elect_one(), do_rows = operand(base + Smem::kDo, 16);
        uint32_t phase = 0, pos = 0;
        for (uint32_t r = 0;; ++r) {
            const QueryWork it = make_queries(a, feed_next<false>(sh.feed, r, failed));
            if (!it.valid) break;
            auto products_of = [&](int32_t j, uint32_t b) {
                const uint32_t stage = (pos + j) % kValueStages;
                bar_wait(full + 8 * (kKeyStages + stage), (pos + j) / kValueStages & 1, failed);
                fence_after();
                product_of_rows<Q, D>(lead, tmem + kTile + b * kTile, do_rows, operand(base + Smem::kValues + stage * Smem::kTileBytes, 16), it.seen(j));
                mma_commit(lead, products + 8 * b);
                mma_commit(lead, empty + 8 * (kKeyStages + stage));
                if (j + 1 == it.n) mma_commit(lead, queries_free);
            };
            bar_wait(queries, r & 1, failed);
#pragma unroll 1
            for (int32_t j = -2; j < it.n; ++j) {
                const uint32_t b = j & 1;
                if (j >= 0) {
                    const uint32_t stage = (pos + j) % kKeyStages, at = base + Smem::kKeys + stage * Smem::kTileBytes;
                    const int32_t count = it.count(j), seen = it.seen(j);
                    bar_wait(full + 8 * stage, (pos + j) / kKeyStages & 1, failed);
                    if ((count & 15) && seen > (count & ~15)) {
                        clear_rows<D>(at, count);
                        publish_clears();
                    }
                    bar_wait(gradients + 8 * b, phase >> b & 1, failed);
                    phase ^= 1u << b;
                    if (j == 0 && r > 0) bar_wait(sums_free, (r + 1) & 1, failed);
                    fence_after();
                    const uint32_t ds = tmem + kTile + b * kTile, k_columns = operand(at, kTile * 128);
                    product_with_weights<Q, D>(lead, tmem + 3 * kTile, ds, k_columns, seen, j == 0);
                    product_with_weights<Q, D>(lead, tmem + 3 * kTile, ds + kRest, k_columns, seen, false);
                    mma_commit(lead, empty + 8 * stage);
                    if (j + 1 == it.n) mma_commit(lead, sums);
                }
                if (j + 2 < it.n) products_of(j + 2, b);
            }
            pos += it.n;
        }
    } else if (warp < 8) {
        const int half = warp >> 2, row = threadIdx.x & (kTile - 1);
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
        const uint32_t t_s = lanes + half * kHalfTile;
        const int32_t row_token = row / a.hp, row_head = row - row_token * a.hp;
        const float c = exp2f((float)(shift - up));
        const float2 scale2 = make_float2(a.scale_log2, a.scale_log2), c2 = make_float2(c, c);
        auto stats_of = [&](const QueryWork &w) {
            float2 st = make_float2(INFINITY, 0.f);
            if (w.valid && row_token < w.tokens && HORA_IN(w.token0 + row_token, a.T)) st = __ldcg(reinterpret_cast<const float2 *>(a.stats + (int64_t)(w.token0 + row_token) * a.Hq + w.block * a.hp + row_head));
            return st;
        };
        uint32_t phase = 0, products_phase = 0;
        for (int32_t r = 0; ok; ++r) {
            const QueryWork it = make_queries(a, feed_next<false>(sh.feed, r, failed));
            if (!it.valid) break;
            const int64_t row_at = (int64_t)(it.token0 + row_token) * a.Hq + it.block * a.hp + row_head;
            const float2 st = stats_of(it);
            const float2 lse2 = make_float2((float)up - st.x, (float)up - st.x), delta2 = make_float2(-st.y * c, -st.y * c);
            const bool have = row_token < it.tokens && HORA_IN(it.token0 + row_token, a.T);
            const int32_t token = it.token0 + row_token;
            const int32_t seen_to = a.causal && have ? min(it.end, token + 1) : it.end;
            float2 off = make_float2(0.f, 0.f);
            for (int32_t j = 0; j < it.n; ++j, phase ^= 1) {
                const int32_t limit = (j < it.n_shared ? it.shared1 - it.shared0 - j * kTile : seen_to - it.own0 - (j - it.n_shared) * kTile) - half * kHalfTile;
                ok = bar_wait(scores, phase, failed);
                ok = __all_sync(kFull, ok);
                if (!ok) break;
                fence_after();
                float p[2][32];
#pragma unroll
                for (int b = 0; b < 2; ++b) tmem_load(t_s + b * 32, p[b]);
                tmem_load_wait();
                fence_before();
                bar_arrive(scores_free);
                const bool border = __any_sync(kFull, limit < kHalfTile);
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float2 y = fma2(make_float2(p[b][e], p[b][e + 1]), scale2, lse2);
                        p[b][e] = exp2_approx(y.x);
                        p[b][e + 1] = exp2_approx(y.y);
                    }
                const uint32_t b2 = j & 1, t_dp = lanes + kTile + b2 * kTile + half * kHalfTile;
                ok = bar_wait(products + 8 * b2, products_phase >> b2 & 1, failed);
                products_phase ^= 1u << b2;
                ok = __all_sync(kFull, ok);
                if (!ok) break;
                fence_after();
                float dp[2][32];
#pragma unroll
                for (int b = 0; b < 2; ++b) tmem_load(t_dp + b * 32, dp[b]);
                tmem_load_wait();
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    uint32_t w[8], rest[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float *x = p[b >> 1] + (b & 1) * 16 + 2 * e, *d = dp[b >> 1] + (b & 1) * 16 + 2 * e;
                        float2 y = mul2(make_float2(x[0], x[1]), fma2(make_float2(d[0], d[1]), c2, delta2));
                        if (border) {                    // keys of others may hold anything
                            if (b * 16 + 2 * e >= limit) y.x = 0.f;
                            if (b * 16 + 2 * e + 1 >= limit) y.y = 0.f;
                        }
                        off = add2(off, y);
                        w[e] = pack2(y.x, y.y, Q());
                        const float2 held = unpack2(w[e], Q());
                        rest[e] = pack2(y.x - held.x, y.y - held.y, Q());
                    }
                    tmem_store8(t_dp + b * 8, w);
                    tmem_store8(t_dp + kRest + b * 8, rest);
                }
                tmem_store_wait();
                fence_before();
                bar_arrive(gradients + 8 * b2);
            }
            if (!ok) break;
            // a row's dS add up to nothing; what they add up to is what dout . out was off by
            if (have && ok) (half ? a.stats[row_at].w : a.stats[row_at].z) = (off.x + off.y) * exp2f((float)-shift);
            ok = bar_wait(sums, r & 1, failed);
            ok = __all_sync(kFull, ok);
            if (!ok) break;
            fence_after();
            store_row<D / 2>(static_cast<Q *>(a.dq) + (int64_t)token * a.dq_stride + (int64_t)(it.block * a.hp + row_head) * D + half * (D / 2),
                             lanes + 3 * kTile + half * (D / 2), a.scale * exp2f((float)-shift), have);
            fence_before();
            bar_arrive(sums_free);
        }
    }
    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && sh.failed) raise_status(a.status, HORA_ERR_INTERNAL);
    if (warp == 0) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <typename Q, int D>
hora_status_t launch_backward(const PackedArgs &a, const void *q, const void *k, const void *v, int64_t q_stride, int32_t dtype, cudaStream_t stream) {
    CUtensorMap q_map, do_map, k_map, v_map;
    if (!head_map(&q_map, q, dtype, D, a.Hq, a.T, q_stride, a.hp, a.tp) || !head_map(&do_map, a.dout, dtype, D, a.Hq, a.T, a.dout_stride, a.hp, a.tp) ||
        !head_map(&k_map, k, dtype, D, a.Hkv, a.T, a.k_stride, 1, kTile) || !head_map(&v_map, v, dtype, D, a.Hkv, a.T, a.v_stride, 1, kTile))
        return HORA_ERR_CUDA;
    constexpr int kKeysSmem = KeysSmem<D>::kSmall + (int)sizeof(KeysShared), kQueriesSmem = QueriesSmem<D>::kSmall + (int)sizeof(QueriesShared);
    static std::atomic<uint64_t> keys_devices{0}, queries_devices{0};
    cudaError_t e = allow_shared(reinterpret_cast<const void *>(packed_keys_kernel<Q, D>), kKeysSmem, keys_devices);
    if (e == cudaSuccess) e = allow_shared(reinterpret_cast<const void *>(packed_queries_kernel<Q, D>), kQueriesSmem, queries_devices);
    if (e == cudaSuccess)
        e = launch_pdl(packed_queries_kernel<Q, D>, clamp_grid((int64_t)a.query_cap * a.blocks, 1), kPackedThreads, kQueriesSmem, stream, a, q_map, do_map, k_map, v_map);
    if (e == cudaSuccess)
        e = launch_pdl(packed_keys_kernel<Q, D>, clamp_grid(((int64_t)a.T / kTile + a.S) * a.Hkv + 2 * a.n_sm, 1), kPackedThreads, kKeysSmem, stream, a, q_map, do_map, k_map, v_map);
    count_launches(2);
    return cuda_ok(e);
}

}  // namespace

hora_status_t launch_packed_backward(const PackedArgs &a, const void *q, const void *k, const void *v, int64_t q_stride, int32_t dtype, cudaStream_t stream) {
    if (dtype == HORA_DTYPE_BF16)
        return a.D == 128 ? launch_backward<__nv_bfloat16, 128>(a, q, k, v, q_stride, dtype, stream) : launch_backward<__nv_bfloat16, 64>(a, q, k, v, q_stride, dtype, stream);
    return a.D == 128 ? launch_backward<__half, 128>(a, q, k, v, q_stride, dtype, stream) : launch_backward<__half, 64>(a, q, k, v, q_stride, dtype, stream);
}

}  // namespace hora
