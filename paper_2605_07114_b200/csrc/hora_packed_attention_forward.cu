// hora_packed_attention: the forward kernel.
//
// Per row: m a reference near the running maximum of s = scale q.k (in units of log2), l = sum 2^(s - m), o = sum 2^(s - m) v;  out = o / l,
// lse = m ln 2 + log l.  A CTA holds an SM and works on two tiles of 128 query rows at a time, which share the keys and values.
// Each tile has four warps for its softmax, one thread to a row, and one that issues its products; one more warp brings in queries, keys and
// values by TMA, and four read, norm and store outputs while the next item is under way.  S = Q K^T is accumulated in tensor memory, 64 keys
// at a time in two places in turn, so that the next scores are there while a softmax works on these; the weights P replace them in 16
// bits (rounded once, as the product needs them; sums are of the unrounded ones) and are the left operand of O += P V.
//   O is scaled only when a row's maximum has grown by more than 2^8 (weights up to 256 are as exact as weights up to 1), after the product
// before has been waited for.
//   fp16 has only 2^-14 below 1 at full precision and nothing below 2^-25, where rows with one dominant key of little value live on their small
// weights (a key 16 above the others' mean score among 16381: 6 % off).  There weights are held times 2^7, the most with which none passes 2^15: m is
// that much below the maximum when it is set.  (2^10, as in the backward pass, leaves a maximum only 2^4 to grow by before O has to be scaled: 5 % more
// time for scores of a deviation of 2.)  bf16 has fp32's exponents.
//   Keys that are not of the sequence are in no row's sum; the product stops at the last sixteen that hold one of it, and values
// of others among those are cleared in shared memory first, since 0 * NaN is not 0.
//   The warps of a multiprocessor share its instruction cache, and those that issue the products wait for their instructions longest: the code is
// kept small (waits that were unrolled, 165 KB in all, cost a quarter of the time).
//   What bounds it: power for one long document (16381 tokens of 32 heads of 128: 1.9 to 2.2 ms, 1000 to 1160 TFLOP/s); else the chain scores -
// maximum - weights - product of its eight softmax warps, 1.3 thousand cycles for 64 keys of both tiles (exponentials alone take 1.0), and
// the way of the next queries into shared memory (60 prompts up to 509 tokens: 114 us and 0.57 PFLOP/s where inputs stay from pass to pass, 136 where
// they change; 15 groups of 32 rollouts: 1.1 ms and 0.78 PFLOP/s, 1.25 to 1.3 ms).  64 keys at a time because the next scores are then there when a softmax is through (128 at a time: 137 us for the 60
// prompts), although a product of 64 keys takes the tensor cores as long as one of 128.
//   Every wait has a limit; a wait that reaches it makes the CTA give up and report HORA_ERR_INTERNAL.
#define HORA_FILE_ID 11
#include <type_traits>

#include "hora_packed_attention.cuh"

HORA_CHECKED_REGISTER()

namespace hora {

namespace {

constexpr int kTile = kPackedRows, kHalfTile = kTile / 2;
constexpr int kForwardThreads = 512;
constexpr int kLoadWarp = 8, kProductWarp = 9, kFeedWarp = 11, kOutputWarp = 12;      // the first 8: softmax; two: products; from 12 on: outputs
constexpr int kFeedReaders = 15;                         // warps that take items from the feeder

template <int D>
struct ForwardSmem {
    static constexpr int kTileBytes = kTile * D * 2;
    static constexpr int kStages = D == 128 ? 4 : 8;
    static constexpr int kQ = 0, kRing = 2 * kTileBytes, kStaging = kRing + kStages * kTileBytes;        // staging: 32 rows of 64 bytes a warp
    static constexpr int kSmall = kStaging + 4 * kWarp * 64;
};

struct ForwardShared {
    Feed feed;
    float2 sums[2][kTile];                               // of a tile's rows: m, l
    uint64_t full[8], empty[8], queries, queries_free, scores[4], weights[4], product[2], output[2], output_free[2], summed[2], sums_free[2];
    int32_t failed;
    uint32_t tmem;
};

// An item as the warps need it: runs of keys, steps of each tile.
struct Item {
    int32_t token0, end, own0, shared0, shared1;
    int32_t block;
    int32_t n_shared, n[2], tokens[2], last[2];          // last: behind the last key that the tile sees of its own sequence

    __device__ __forceinline__ int32_t steps() const { return max(n[0], n[1]); }
    // first key of step j and how many keys of the sequence there are from it on; and those that tile t sees
    __device__ __forceinline__ int32_t key0(int32_t j) const { return j < n_shared ? shared0 + j * kTile : own0 + (j - n_shared) * kTile; }
    __device__ __forceinline__ int32_t count(int32_t j) const { return min(kTile, (j < n_shared ? shared1 : end) - key0(j)); }
    __device__ __forceinline__ int32_t seen(int32_t j, int t) const { return min(kTile, (j < n_shared ? shared1 : t ? last[1] : last[0]) - key0(j)); }
};

__device__ __forceinline__ Item make_item(const PackedArgs &a, const FeedSlot &f) {
    Item q;
    q.token0 = f.a.x;
    q.own0 = f.a.z;
    q.end = f.a.w;
    q.shared0 = f.b.x;
    q.shared1 = f.b.y;
    q.block = f.part;
    q.n_shared = (q.shared1 - q.shared0 + kTile - 1) / kTile;
    q.tokens[0] = min(a.tp, f.a.y);
    q.tokens[1] = f.a.y - q.tokens[0];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        q.last[t] = a.causal ? q.token0 + t * a.tp + q.tokens[t] : q.end;
        q.n[t] = q.tokens[t] > 0 ? q.n_shared + (q.last[t] - q.own0 + kTile - 1) / kTile : 0;
    }
    return q;
}

// How far below a row's maximum its reference lies when it is set.
template <typename Q>
constexpr float kBelow = std::is_same<Q, __half>::value ? 7.f : 0.f;

// A row's part in 64 keys: scores in tensor memory, of which the row sees `limit`, to weights there; `whole`: every row of the warp sees all.
// `have`: the row is a token's; others may hold anything and have no say.  `first`: there is no output yet; else `before` tells that the product
// before is in.
template <typename Q, int D>
__device__ __forceinline__ bool softmax_step(uint32_t t_s, uint32_t t_o, float scale_log2, int32_t limit, bool whole, bool have, bool first, uint32_t before,
                                             uint32_t before_phase, float &m, float &l, volatile int32_t *failed) {
    float s[2][32], top[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) tmem_load(t_s + b * 32, s[b]);
    tmem_load_wait();
    if (!whole) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int32_t n = limit - b * 32;
            const uint32_t sees = n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u;
#pragma unroll
            for (int e = 0; e < 32; ++e)
                if (!(sees & (1u << e))) s[b][e] = -INFINITY;
        }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        top[b] = s[b][0];
#pragma unroll
        for (int e = 1; e < 31; e += 2) top[b] = fmaxf(top[b], fmaxf(s[b][e], s[b][e + 1]));
        top[b] = fmaxf(top[b], s[b][31]);
    }
    top[0] = fmaxf(top[0], top[1]) * scale_log2;
    // beyond 2^22 differences of scores are rounded by so much that weights need the room themselves
    const float below = kBelow<Q> > 0.f && fabsf(top[0]) < 4194304.f ? kBelow<Q> : 0.f;
    if (first) {
        m = top[0] - below;
    } else if (__any_sync(kFull, have && top[0] > m + (below + 8.f))) {
        if (!__all_sync(kFull, bar_wait(before, before_phase, failed))) return false;
        fence_after();
        const float up = fmaxf(m, top[0] - below), f = up == -INFINITY ? 1.f : exp2_approx(m - up);
        l *= f;
        m = up;
#pragma unroll 1
        for (int b = 0; b < D / 16; ++b) {
            float o[16];
            tmem_load16(t_o + b * 16, o);
            tmem_load_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= f;
            tmem_store16(t_o + b * 16, o);
        }
    }
    // where no key has been seen the reference is -infinity and every weight has to come out as 0
    const float z = m == -INFINITY ? 0.f : m;
    const float2 scale2 = make_float2(scale_log2, scale_log2), z2 = make_float2(-z, -z);
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int b = 0; b < 4; ++b) {                        // sixteen at a time, in place of scores that have been read
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float2 y = fma2(make_float2(s[b >> 1][(b & 1) * 16 + 2 * e], s[b >> 1][(b & 1) * 16 + 2 * e + 1]), scale2, z2);
            y = make_float2(exp2_approx(y.x), exp2_approx(y.y));
            sum = add2(sum, y);
            w[e] = pack2(y.x, y.y, Q());
        }
        tmem_store8(t_s + b * 8, w);
    }
    l += sum.x + sum.y;
    tmem_store_wait();
    fence_before();
    return true;
}

extern __shared__ __align__(1024) uint8_t s_forward[];

template <typename Q, int D>
__global__ void __launch_bounds__(kForwardThreads, 1)
packed_forward_kernel(const PackedArgs a, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                      const __grid_constant__ CUtensorMap v_map) {
    using Smem = ForwardSmem<D>;
    constexpr int kStages = Smem::kStages, kParts = D / 64;
    ForwardShared &sh = *reinterpret_cast<ForwardShared *>(s_forward + Smem::kSmall);
    const uint32_t base = smem_at(s_forward);
    const int warp = threadIdx.x >> 5, lane = lane_id();
    volatile int32_t *failed = &sh.failed;
    if (base & 1023u) {
        pdl_enter();
        raise_status(a.status, HORA_ERR_INTERNAL);
        return;
    }
    const uint32_t full = smem_at(sh.full), empty = smem_at(sh.empty), queries = smem_at(&sh.queries), queries_free = smem_at(&sh.queries_free),
                   product = smem_at(sh.product), scores = smem_at(sh.scores), weights = smem_at(sh.weights), output = smem_at(sh.output), output_free = smem_at(sh.output_free),
                   summed = smem_at(sh.summed), sums_free = smem_at(sh.sums_free);
    if (threadIdx.x == 0) {
        sh.failed = 0;
        feed_init(sh.feed, kFeedReaders);
        for (int s = 0; s < kStages; ++s) {
            bar_init(full + 8 * s, 1);
            bar_init(empty + 8 * s, 2);                  // both tiles' products
        }
        bar_init(queries, 1);
        bar_init(queries_free, 2);
        for (int t = 0; t < 2; ++t) {
            for (int h = 0; h < 2; ++h) {
                bar_init(scores + 16 * t + 8 * h, 1);
                bar_init(weights + 16 * t + 8 * h, kTile);
            }
            bar_init(product + 8 * t, 1);
            bar_init(output + 8 * t, 1);
            bar_init(output_free + 8 * t, kTile);
            bar_init(summed + 8 * t, kTile);
            bar_init(sums_free + 8 * t, kTile);
        }
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
    const uint32_t tmem = sh.tmem;                       // columns: S of the two tiles, 128 each, then O, D each
    pdl_enter();
    bool ok = true;

    if (warp >= kOutputWarp) {
        // ---- outputs of the two tiles, while the next item is under way
        const int row = threadIdx.x & (kTile - 1);
        const int32_t row_token = row / a.hp, row_head = row - row_token * a.hp;
        uint32_t phase = 0;                              // a bit for each tile
        for (uint32_t r = 0; ok; ++r) {
            const FeedSlot f = feed_next<false>(sh.feed, r, failed);
            if (!f.valid) break;
            const Item it = make_item(a, f);
            const int32_t head = it.block * a.hp + row_head;
#pragma unroll 1
            for (int t = 0; t < 2; ++t) {
                const int32_t tokens = t ? it.tokens[1] : it.tokens[0];
                if (tokens == 0) continue;
                const int32_t token = it.token0 + t * a.tp + row_token;
                const bool have = row_token < tokens && HORA_IN(token, a.T);
                ok = bar_wait(summed + 8 * t, phase >> t & 1, failed);
                const float2 ml = sh.sums[t][row];
                bar_arrive(sums_free + 8 * t);
                const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;        // NaN where a score was NaN: it is in no maximum, but in the sum
                constexpr float kSum = std::is_same<Q, __half>::value ? 1.f / 128.f : 1.f;      // 2^-kBelow
                if (have && ok && a.lse != nullptr) a.lse[(int64_t)token * a.Hq + head] = (ml.x == -INFINITY ? 0.f : kLn2 * (ml.x + kBelow<Q>)) + logf(ml.y * kSum);
                ok = ok && bar_wait(output + 8 * t, phase >> t & 1, failed);
                phase ^= 1u << t;
                ok = __all_sync(kFull, ok);
                if (!ok) break;
                fence_after();
                const uint32_t t_o = tmem + ((uint32_t)(warp & 3) << 21) + 256 + t * D;
                const int64_t to = have ? (int64_t)token * a.out_stride + (int64_t)head * D : -1;
                // 32 columns at a time through shared memory, so that four lanes store 64 bytes of a row
                const uint32_t staging = base + Smem::kStaging + (warp & 3) * (kWarp * 64);
                int64_t at[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) at[v] = __shfl_sync(kFull, to, v * 8 + (lane >> 2));
#pragma unroll 1
                for (int p = 0; p < D / 32; ++p) {
                    float o[32];
                    tmem_load(t_o + p * 32, o);
                    tmem_load_wait();
                    if (p == D / 32 - 1) {
                        fence_before();
                        bar_arrive(output_free + 8 * t);
                    }
                    __syncwarp();
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = o[v * 8 + e] * inv;
                        const uint4 y = pack8<Q>(x);
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(staging + lane * 64 + ((v ^ (lane >> 1 & 3)) << 4)), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w) : "memory");
                    }
                    __syncwarp();
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int x = v * 8 + (lane >> 2);   // row of the warp
                        uint4 y;
                        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(y.x), "=r"(y.y), "=r"(y.z), "=r"(y.w) : "r"(staging + x * 64 + (((lane & 3) ^ (x >> 1 & 3)) << 4)) : "memory");
                        if (at[v] >= 0) *reinterpret_cast<uint4 *>(static_cast<Q *>(a.out) + at[v] + p * 32 + (lane & 3) * 8) = y;
                    }
                }
            }
        }
    } else if (warp >= 8) {
        if (warp == kFeedWarp) {
            if (lane == 0) feed<2>(sh.feed, reinterpret_cast<const int4 *>(a.query_items), __ldcg(a.counts), a.query_cap, a.blocks, a.counts + 4, failed);
        } else if (warp == kLoadWarp) {
            if (lane == 0) {
                int32_t pos = 0;                         // copies into the ring so far
                uint32_t r = 0;
                for (; ok; ++r) {
                    const FeedSlot f = feed_next<true>(sh.feed, r, failed);
                    if (!f.valid) break;
                    const Item it = make_item(a, f);
                    const int32_t head = it.block * a.hp / a.g;
                    const int tiles = it.tokens[1] > 0 ? 2 : 1;
                    if (r > 0) ok = bar_wait(queries_free, (r + 1) & 1, failed);
                    if (!ok) break;
                    bar_expect(queries, tiles * kParts * a.hp * a.tp * 128);
                    for (int t = 0; t < tiles; ++t)
                        for (int p = 0; p < kParts; ++p)
                            tma_box3(base + Smem::kQ + t * Smem::kTileBytes + p * (kTile * 128), &q_map, p * 64, it.block * a.hp, it.token0 + t * a.tp, queries);
                    const int32_t n = it.steps();
                    for (int32_t j = 0; j < n && ok; ++j)
                        for (int which = 0; which < 2; ++which, ++pos) {
                            const int stage = pos % kStages;
                            if (pos >= kStages) ok = bar_wait(empty + 8 * stage, (pos / kStages + 1) & 1, failed);
                            if (!ok) break;
                            bar_expect(full + 8 * stage, Smem::kTileBytes);
                            for (int p = 0; p < kParts; ++p)
                                tma_box3(base + Smem::kRing + stage * Smem::kTileBytes + p * (kTile * 128), which ? &v_map : &k_map, p * 64, head, it.key0(j), full + 8 * stage);
                        }
                }
                // the CTA may not end while copies are on their way to it: each is waited for by its use, unless the CTA has given up
                if (*failed) {
                    int32_t never = 0;
                    for (int32_t x = max(0, pos - kStages); x < pos; ++x) bar_wait(full + 8 * (x % kStages), (x / kStages) & 1, &never);
                    if (r > 0) bar_wait(queries, (r - 1) & 1, &never);
                }
            }
        } else {
            // ---- products of one tile.  A wait that has failed is not looked at here: what follows is of no use, but in bounds, and there is no
            // next item
            const int t = warp - kProductWarp;
            const uint32_t lead = elect_one();
            constexpr uint32_t kType = std::is_same<Q, __nv_bfloat16>::value ? 1u : 0u;
            constexpr uint32_t kIdescS = (1u << 4) | (kType << 7) | (kType << 10) | ((kTile / 16) << 24);      // and the columns / 8 at bit 17
            constexpr uint32_t kIdescO = (1u << 4) | (kType << 7) | (kType << 10) | (1u << 16) | ((D / 8) << 17) | ((kTile / 16) << 24);
            const uint32_t k_ring = operand(base + Smem::kRing, 16), v_ring = operand(base + Smem::kRing, kTile * 128);
            const uint32_t q = operand(base + Smem::kQ + t * Smem::kTileBytes, 16), t_s = tmem + t * kTile, t_o = tmem + 256 + t * D;
            const uint32_t told = weights + 16 * t;
            uint32_t weights_phase = 0, outputs = 0, pos = 0;
            // every copy is waited for, used or not: a barrier only tells two neighbouring ones apart
            auto arrived = [&](uint32_t x) { bar_wait(full + 8 * (x % kStages), (x / kStages) & 1, failed); };
            for (uint32_t r = 0;; ++r) {
                const FeedSlot f = feed_next<false>(sh.feed, r, failed);
                if (!f.valid) break;
                const Item it = make_item(a, f);
                const int32_t n = it.steps(), mine = t ? it.n[1] : it.n[0];
                int32_t js = 0, hs = 0;                  // the next scores': step and half
                auto scores_of = [&](uint32_t b) {
                    const uint32_t x = pos + 2 * js;
                    if (hs == 0) arrived(x);
                    const int32_t seen = it.seen(js, t) - hs * kHalfTile;
                    const uint32_t k = k_ring + x % kStages * (Smem::kTileBytes >> 4) + hs * (kHalfTile * 128 >> 4), to = t_s + b * kHalfTile;
                    const uint32_t idesc = kIdescS | (uint32_t)((min(seen, kHalfTile) + 15) >> 4) << 18;
                    fence_after();
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) {
                        const uint32_t off = ((x >> 2) * (kTile * 128) + (x & 3) * 32) >> 4;
                        mma_smem(lead, to, q + off, k + off, idesc, x > 0);
                    }
                    mma_commit(lead, scores + 16 * t + 8 * b);
                    if (hs == 0 && seen > kHalfTile) {
                        hs = 1;
                    } else {
                        mma_commit(lead, empty + 8 * (x % kStages));
                        hs = 0;
                        if (++js == mine) mma_commit(lead, queries_free);
                    }
                };
                bar_wait(queries, r & 1, failed);
                if (mine == 0) mma_commit(lead, queries_free);
                uint32_t i = 0;
                int32_t seen = 0;
#pragma unroll 1
                for (int32_t j = 0, h = 0; j < mine; ++i) {
                    // scores are two halves ahead of the product
                    if (i == 0) {
                        scores_of(0);
                        if (js < mine) scores_of(1);
                    }
                    const uint32_t b = i & 1, x = pos + 2 * j + 1;
                    if (h == 0) {
                        arrived(x);
                        seen = it.seen(j, t);
                    }
                    const int32_t count = it.count(j);
                    if (count < min((h + 1) * kHalfTile, (seen + 15) & ~15) && count > h * kHalfTile) {        // values that are not of the sequence, among the last sixteen
                        const uint32_t at = base + Smem::kRing + x % kStages * Smem::kTileBytes;
                        const int32_t clear = ((count + 15) & ~15) - count;
                        for (int32_t c = lane; c < clear * (D / 8); c += kWarp) {
                            const uint32_t to = at + (c % (D / 8) >> 3) * (kTile * 128) + (count + c / (D / 8)) * 128 + (c & 7) * 16;
                            asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(to), "r"(0) : "memory");
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    bar_wait(told + 8 * b, weights_phase >> b & 1, failed);
                    weights_phase ^= 1u << b;
                    if (i == 0) {                        // the output of the item before has been read
                        if (outputs > 0) bar_wait(output_free + 8 * t, (outputs + 1) & 1, failed);
                        ++outputs;
                    }
                    fence_after();
                    const uint32_t v = v_ring + x % kStages * (Smem::kTileBytes >> 4) + h * (kHalfTile * 128 >> 4), w = t_s + b * kHalfTile;
                    const int32_t left = seen - h * kHalfTile;
                    mma_tmem(lead, t_o, w, v, kIdescO, i > 0);
                    if (left >= kHalfTile) {
#pragma unroll
                        for (int g = 1; g < 4; ++g) mma_tmem(lead, t_o, w + g * 8, v + g * (2048 >> 4), kIdescO, 1);
                    } else {
#pragma unroll 1
                        for (int g = 1; g * 16 < left; ++g) mma_tmem(lead, t_o, w + g * 8, v + g * (2048 >> 4), kIdescO, 1);
                    }
                    mma_commit(lead, product + 8 * t);
                    if (h == 0 && left > kHalfTile) {
                        h = 1;
                    } else {
                        mma_commit(lead, empty + 8 * (x % kStages));
                        h = 0;
                        if (++j == mine) mma_commit(lead, output + 8 * t);
                    }
                    if (js < mine) scores_of(b);
                }
                for (int32_t j = mine; j < n; ++j)
                    for (uint32_t x = pos + 2 * j; x < pos + 2 * j + 2; ++x) {
                        arrived(x);
                        mma_commit(lead, empty + 8 * (x % kStages));
                    }
                pos += 2 * n;
            }
        }
    } else {
        // ---- softmax: thread `row` of a tile has row `row` of its scores
        const int t = warp >> 2, row = threadIdx.x & (kTile - 1);
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
        const uint32_t t_s = lanes + t * kTile, t_o = lanes + 256 + t * D;
        const int32_t row_token = row / a.hp;
        uint32_t scores_phase = 0, ended = 0, products = 0;                    // products of all items before
        for (uint32_t r = 0; ok; ++r) {
            const FeedSlot f = feed_next<false>(sh.feed, r, failed);
            if (!f.valid) break;
            const Item it = make_item(a, f);
            const int32_t n = t ? it.n[1] : it.n[0], tokens = t ? it.tokens[1] : it.tokens[0];
            if (n == 0) continue;
            const int32_t token = it.token0 + t * a.tp + row_token;
            const bool have = row_token < tokens;
            const int32_t seen_to = a.causal && have ? min(it.end, token + 1) : it.end;
            float m = -INFINITY, l = 0.f;
            uint32_t i = 0;
            for (int32_t j = 0, h = 0; j < n; ++i) {
                // keys of the half that the row sees
                const int32_t limit = (j < it.n_shared ? it.shared1 - it.shared0 - j * kTile : seen_to - it.own0 - (j - it.n_shared) * kTile) - h * kHalfTile;
                const uint32_t b = i & 1;
                ok = bar_wait(scores + 16 * t + 8 * b, scores_phase >> b & 1, failed);
                scores_phase ^= 1u << b;
                ok = __all_sync(kFull, ok);
                if (!ok) break;
                fence_after();
                ok = softmax_step<Q, D>(t_s + b * kHalfTile, t_o, a.scale_log2, limit, !__any_sync(kFull, limit < kHalfTile), have, i == 0, product + 8 * t,
                                        (products + i - 1) & 1, m, l, failed);
                if (!ok) break;
                bar_arrive(weights + 16 * t + 8 * b);
                if (h == 0 && it.seen(j, t) > kHalfTile) {
                    h = 1;
                } else {
                    h = 0;
                    ++j;
                }
            }
            products += i;
            if (!ok) break;
            if (ended > 0) ok = bar_wait(sums_free + 8 * t, (ended + 1) & 1, failed);
            ++ended;
            ok = __all_sync(kFull, ok);
            if (!ok) break;
            sh.sums[t][row] = make_float2(m, l);
            bar_arrive(summed + 8 * t);
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
hora_status_t launch_forward(const PackedArgs &a, const void *q, const void *k, const void *v, int64_t q_stride, int32_t dtype, cudaStream_t stream) {
    CUtensorMap q_map, k_map, v_map;
    if (!head_map(&q_map, q, dtype, D, a.Hq, a.T, q_stride, a.hp, a.tp) || !head_map(&k_map, k, dtype, D, a.Hkv, a.T, a.k_stride, 1, kTile) ||
        !head_map(&v_map, v, dtype, D, a.Hkv, a.T, a.v_stride, 1, kTile))
        return HORA_ERR_CUDA;
    constexpr int kSmem = ForwardSmem<D>::kSmall + (int)sizeof(ForwardShared);
    static std::atomic<uint64_t> devices{0};
    cudaError_t e = allow_shared(reinterpret_cast<const void *>(packed_forward_kernel<Q, D>), kSmem, devices);
    const int64_t most = (int64_t)a.query_cap * a.blocks;
    if (e == cudaSuccess) e = launch_pdl(packed_forward_kernel<Q, D>, clamp_grid(most, 1), kForwardThreads, kSmem, stream, a, q_map, k_map, v_map);
    count_launches(1);
    return cuda_ok(e);
}

}  // namespace

hora_status_t launch_packed_forward(const PackedArgs &a, const void *q, const void *k, const void *v, int64_t q_stride, int32_t dtype, cudaStream_t stream) {
    if (dtype == HORA_DTYPE_BF16)
        return a.D == 128 ? launch_forward<__nv_bfloat16, 128>(a, q, k, v, q_stride, dtype, stream) : launch_forward<__nv_bfloat16, 64>(a, q, k, v, q_stride, dtype, stream);
    return a.D == 128 ? launch_forward<__half, 128>(a, q, k, v, q_stride, dtype, stream) : launch_forward<__half, 64>(a, q, k, v, q_stride, dtype, stream);
}

}  // namespace hora
