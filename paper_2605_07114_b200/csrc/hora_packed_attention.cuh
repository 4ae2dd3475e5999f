// hora_packed_attention and its backward pass: what their kernels share.
//
// The packed tokens hold S sequences one after the other.  A query sees keys of its own sequence and, where that is a rollout, its group's
// prompt, the sequence in front of the group's rollouts.  Both are runs of tokens, and in the causal case "sees" is: the key
// lies in one of the two runs and not behind the query.  Seen from a key: the queries are one run, from the key to the end of its
// sequence, or of its group if it is of a prompt.
//   A tile of queries is tp tokens times hp heads of one cache head's g (hp divides g, hp * tp <= 128): all of them read the same keys.
// Few tokens to a tile mean that the causal border cuts off little of it, and short sequences fill it.  A plan lists the tiles by
// falling number of steps; CTAs, one to an SM, take them from a counter, the longest first, so that none ends much later than the others.
#pragma once

#include "hora_checked.cuh"
#include "hora_rows16.cuh"
#include "hora_tensor.cuh"

namespace hora {

constexpr int kPackedRows = 128;                         // rows of a tile, keys of a step
constexpr int kPackedThreads = 384;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Tokens whose queries are an item, their sequence's begin and end, and the prompt's.
struct QueryItem {
    int32_t token0, tokens, own0, end, shared0, shared1, pad[2];
};
// Keys that are an item, and the run of tokens whose queries may see them; or a part of that run (of a prompt's keys under a large group), whose
// sums are then left in 32 bits in the slots slot0 + part (times heads), and added up, in order, by those that come last to
// the item's tickets.
struct KeyItem {
    int32_t key0, keys, q0, q1, slot0, parts, part, ticket;
};

struct PackedArgs {
    const int64_t *seq_offsets, *group_offsets;
    const void *out_in, *dout, *v;                       // of the backward pass's first kernel
    void *out, *dq, *dk, *dv;
    float *lse;
    int32_t *status;
    int64_t out_stride, dout_stride, k_stride, v_stride, dq_stride, dk_stride, dv_stride;
    int32_t S, N, T, Hq, Hkv, D, g, hp, tp, blocks;       // blocks: of hp heads, of all query heads
    int32_t causal, half;                                // half: fp16 (weights and gradients of scores are held relative to a scale, see below)
    float scale, scale_log2;
    int32_t tile_tokens;                                 // tokens of a query item
    int32_t query_cap, key_cap, n_sm;
    // workspace
    int32_t *counts;                                     // query items, key items, bits of the largest |dout row|^2 and |v row|^2, items taken of either list
    QueryItem *query_items;
    KeyItem *key_items;
    int32_t *tickets;                                    // [n_sm][8]: by warp
    float *slots;                                        // [2 n_sm][dV, dK][128][D]
    float4 *stats;                                       // [T][Hq] (lse in units of log2, dout . out, what that is off by in two parts)
};

// CTAs take the items of a list one after the other, the longest first: the first by their own number, the following ones from a counter.
// One warp (`feeder`) takes them and passes them on to the CTA's other warps through a ring in shared memory, a few items ahead.
constexpr int kFeedDepth = 3;
struct FeedSlot {
    int4 a, b;
    int32_t part, valid, pad[2];                         // which head (or block of heads)
};
struct Feed {
    FeedSlot slot[kFeedDepth];
    uint64_t full[kFeedDepth], empty[kFeedDepth];
};
__device__ __forceinline__ void feed_init(Feed &f, int readers) {
    for (int i = 0; i < kFeedDepth; ++i) {
        bar_init(smem_at(f.full + i), 1);
        bar_init(smem_at(f.empty + i), readers);
    }
}
// One lane.  VECTORS: of 16 bytes an item.
template <int VECTORS>
__device__ __forceinline__ void feed(Feed &f, const int4 *items, int32_t n_items, int32_t cap, int32_t parts, int32_t *taken, volatile int32_t *failed) {
    const int64_t all = (int64_t)n_items * parts;
    for (uint32_t r = 0;; ++r) {
        // the counter cannot pass 2^31: every CTA takes at most one more than there are
        const int64_t x = r == 0 ? blockIdx.x : (int64_t)gridDim.x + (uint32_t)atomicAdd(taken, 1);
        FeedSlot s = {};
        s.valid = x < all && HORA_IN(x / parts, cap);
        if (s.valid) {
            const int64_t i = x / parts;
            s.part = (int32_t)(x - i * parts);
            s.a = __ldcg(items + i * VECTORS);
            if (VECTORS > 1) s.b = __ldcg(items + i * VECTORS + 1);
        }
        const uint32_t at = r % kFeedDepth;
        if (r >= kFeedDepth && !bar_wait(smem_at(f.empty + at), (r / kFeedDepth + 1) & 1, failed)) return;
        f.slot[at] = s;
        bar_arrive(smem_at(f.full + at));
        if (!s.valid) return;
    }
}
// The r-th item of the CTA; by whole warps (ONE: by a single lane, which is then the reader).  Not valid after the last and when the CTA has given up.
template <bool ONE>
__device__ __forceinline__ FeedSlot feed_next(Feed &f, uint32_t r, volatile int32_t *failed) {
    const uint32_t at = r % kFeedDepth;
    bool ok = bar_wait(smem_at(f.full + at), (r / kFeedDepth) & 1, failed);
    if (!ONE) ok = __all_sync(kFull, ok);
    FeedSlot s = {};
    if (ok) {
        s = f.slot[at];
        if (!ONE) __syncwarp();
        if (ONE || lane_id() == 0) bar_arrive(smem_at(f.empty + at));
    }
    return s;
}

// In fp16 the smallest weights and gradients of scores would be lost: weights are held times 2^10, gradients of scores times a power
// of two under which none of them can pass 2^15 (|dS| <= 2 |dout row| |v row|, P <= 1).  bf16 has fp32's exponents: no scale.
constexpr int kHalfShift = 10;
__device__ __forceinline__ int gradient_shift(const PackedArgs &a) {
    if (!a.half) return 0;
    const float d = __int_as_float(__ldcg(a.counts + 2)), v = __int_as_float(__ldcg(a.counts + 3));
    const float bound = 2.f * sqrtf(d) * sqrtf(v);
    if (!(bound > 0.f) || bound > 1e30f) return 0;
    return max(-60, min(60, 14 - ilogbf(bound)));
}

hora_status_t launch_packed_forward(const PackedArgs &a, const void *q, const void *k, const void *v, int64_t q_stride, int32_t dtype, cudaStream_t stream);
hora_status_t launch_packed_backward(const PackedArgs &a, const void *q, const void *k, const void *v, int64_t q_stride, int32_t dtype, cudaStream_t stream);

}  // namespace hora
