// hora_packed_attention: the plan, the first kernel of the backward pass, and the C entries.
#define HORA_FILE_ID 10
#include "hora_packed_attention.cuh"

HORA_CHECKED_REGISTER()

namespace hora {

constexpr int kListThreads = 1024, kListWarps = kListThreads / kWarp;
constexpr int kListBuckets = 1024;                       // of steps: 32 an octave, most first
constexpr int kListOffsets = 4096;                       // group offsets kept in shared memory for the searches

// One sequence: its tokens, the prompt its queries see in front of them, and the end of the queries that see it.
struct PackedSequence {
    int32_t lo, hi, shared0, shared1, seen_to;
};

__device__ __forceinline__ int64_t group_at(const PackedArgs &a, const int64_t *s_groups, int32_t i) { return a.N < kListOffsets ? s_groups[i] : __ldcg(a.group_offsets + i); }

__device__ __forceinline__ int32_t packed_offset(const PackedArgs &a, int64_t i) {
    const int64_t v = __ldcg(a.seq_offsets + i);
    return v < 0 ? 0 : (v > a.T ? a.T : (int32_t)v);
}

__device__ __forceinline__ PackedSequence packed_sequence(const PackedArgs &a, const int64_t *s_groups, int32_t s, bool &bad) {
    PackedSequence q = {0, 0, 0, 0, 0};
    if (s >= a.S) return q;
    const int64_t lo = __ldcg(a.seq_offsets + s), hi = __ldcg(a.seq_offsets + s + 1);
    if (lo < 0 || hi < lo || hi > a.T) bad = true;
    q.lo = packed_offset(a, s);
    q.hi = max(q.lo, packed_offset(a, s + 1));
    q.seen_to = q.hi;
    if (a.group_offsets == nullptr) return q;
    int32_t l = 0, h = a.N;                              // the last group whose prompt is at or before s: group i's is sequence group_offsets[i] + i
    while (h - l > 1) {
        const int32_t mid = (l + h) >> 1;
        if (group_at(a, s_groups, mid) + mid <= s) l = mid;
        else h = mid;
    }
    const int64_t prompt = group_at(a, s_groups, l) + l, last = group_at(a, s_groups, l + 1) + l;
    if (prompt < 0 || last < prompt || last >= a.S || s < prompt || s > last) {
        bad = true;
        return q;
    }
    if (s == prompt) {
        q.seen_to = max(q.hi, packed_offset(a, last + 1));
    } else {
        q.shared0 = packed_offset(a, prompt);
        q.shared1 = min(q.lo, max(q.shared0, packed_offset(a, prompt + 1)));
        if (q.shared1 < q.shared0) q.shared1 = q.shared0;
    }
    return q;
}

__device__ __forceinline__ int32_t steps_of(int32_t n) { return (int32_t)(((int64_t)n + kPackedRows - 1) / kPackedRows); }

// Steps of one item of a sequence; KEYS: of its keys, else of its queries.
template <bool KEYS>
__device__ __forceinline__ int32_t item_steps(const PackedArgs &a, const PackedSequence &q, int32_t i) {
    if constexpr (KEYS) {                                // tiles of queries, for each block of the cache head's query heads
        const int32_t q0 = a.causal ? q.lo + i * kPackedRows : q.lo;
        return (int32_t)(((int64_t)q.seen_to - q0 + a.tp - 1) / a.tp);
    } else {
        const int32_t last = min(q.hi, q.lo + (i + 1) * a.tile_tokens);
        return steps_of(q.shared1 - q.shared0) + steps_of((a.causal ? last : q.hi) - q.lo);
    }
}
template <bool KEYS>
__device__ __forceinline__ int32_t items_of(const PackedArgs &a, const PackedSequence &q) {
    const int32_t per = KEYS ? kPackedRows : a.tile_tokens;
    return (int32_t)(((int64_t)q.hi - q.lo + per - 1) / per);
}
// Parts that an item of keys is cut into: none is longer than what a CTA has to do on average, or than kPartSteps where that is more.
// Parts of items that are cut, times heads, are then 2 n_sm at most: each item has less than n / most + 1 <= 2 n / most of them.
constexpr int kPartSteps = 4;
__device__ __forceinline__ int32_t parts_of(int32_t steps, int32_t most) { return steps > most ? (steps + most - 1) / most : 1; }

__device__ __forceinline__ int32_t bucket_of(int32_t steps) {
    return min(kListBuckets - 1, max(0, kListBuckets - 1 - (int32_t)((__float_as_uint((float)max(1, steps)) >> 18) - (127u << 5))));
}

// f(sequence, item) for all items of 32 * each sequences of a warp's lanes: the items are dealt to the lanes whatever sequence they are of.
// `left`: how many more the warp may take; false, and none taken, where there are more.
template <bool KEYS, typename F>
__device__ __forceinline__ bool for_items(const PackedArgs &a, const PackedSequence &mine, int64_t &left, F f) {
    const int lane = lane_id();
    const int32_t n = items_of<KEYS>(a, mine);
    int64_t upto = n;
#pragma unroll
    for (int d = 1; d < kWarp; d <<= 1) {
        const int64_t o = __shfl_up_sync(kFull, upto, d);
        if (lane >= d) upto += o;
    }
    const int64_t all = __shfl_sync(kFull, upto, kWarp - 1);
    if (all > left) return false;
    left -= all;
    for (int64_t base = 0; base < all; base += kWarp) {
        const int64_t x = base + lane;
        int at = 0;                                      // the first lane whose items reach beyond x
#pragma unroll
        for (int d = kWarp / 2; d > 0; d >>= 1) {
            const int64_t end = __shfl_sync(kFull, upto, at + d - 1);
            if (end <= x) at += d;
        }
        at = min(at, kWarp - 1);
        const int64_t first = __shfl_sync(kFull, upto - n, at);
        PackedSequence q;
        q.lo = __shfl_sync(kFull, mine.lo, at);
        q.hi = __shfl_sync(kFull, mine.hi, at);
        q.shared0 = __shfl_sync(kFull, mine.shared0, at);
        q.shared1 = __shfl_sync(kFull, mine.shared1, at);
        q.seen_to = __shfl_sync(kFull, mine.seen_to, at);
        if (x < all) f(q, (int32_t)(x - first));
    }
    return true;
}

// Lists of items, those with most steps first.  Which of two with about the same number comes first may differ from run to run; results do not.
// Sequences that follow one another have no more items than there are places.  Offsets that are not in order make sequences that overlap, and any
// number of items up to S T: each warp counts its own in 64 bits and stops once they are more than the places, so that neither the counts nor the time
// depend on how many more; the list is then left empty.
template <bool KEYS>
__device__ __forceinline__ void list_items(const PackedArgs &a, const int64_t *s_groups, int32_t *s_bucket, int32_t *s_warp, bool &bad) {
    __shared__ int64_t s_sum[kListWarps];
    __shared__ uint32_t s_items[kListWarps];
    __shared__ int32_t s_next[2];
    const int warp = threadIdx.x >> 5, lane = lane_id();
    const int32_t each = min((int32_t)kWarp, (a.S + kListWarps - 1) / kListWarps);               // sequences of a warp at a time
    const bool once = each * kListWarps >= a.S;
    for (int i = threadIdx.x; i < kListBuckets; i += kListThreads) s_bucket[i] = 0;
    __syncthreads();
    PackedSequence kept = {0, 0, 0, 0, 0};
    const int32_t cap = KEYS ? a.key_cap : a.query_cap;
    int64_t left = cap;
    bool fits = true;
    auto too_many = [&]() {                              // of all warps together, after a barrier; empties the list
        const uint32_t n = s_items[lane];                // 2^31 at most, in two halves whose sums 32 bits hold
        const int64_t all = ((int64_t)__reduce_add_sync(kFull, n >> 16) << 16) + __reduce_add_sync(kFull, n & 0xFFFFu);
        if (all <= cap) return false;
        if (threadIdx.x == 0) a.counts[KEYS ? 1 : 0] = 0;
        bad = true;
        return true;
    };
    int32_t most = 0x7FFFFFFF;
    if constexpr (KEYS) {
        int64_t mine = 0;
        for (int64_t base = (int64_t)warp * each; base < a.S && fits; base += (int64_t)kListWarps * each) {
            kept = lane < each ? packed_sequence(a, s_groups, (int32_t)min((int64_t)a.S, base + lane), bad) : PackedSequence{0, 0, 0, 0, 0};
            fits = for_items<true>(a, kept, left, [&](const PackedSequence &s, int32_t i) { mine += item_steps<true>(a, s, i); });
        }
        if (lane == 0) s_items[warp] = fits ? (uint32_t)(cap - left) : (uint32_t)cap + 1u;
#pragma unroll
        for (int d = kWarp / 2; d > 0; d >>= 1) mine += __shfl_xor_sync(kFull, mine, d);
        if (lane == 0) s_sum[warp] = mine;
        __syncthreads();
        static_assert(kListWarps == kWarp, "a lane to each warp's sum");
        if (too_many()) return;
        int64_t all = s_sum[lane];
#pragma unroll
        for (int d = kWarp / 2; d > 0; d >>= 1) all += __shfl_xor_sync(kFull, all, d);
        const int64_t per = (all * a.Hkv + a.n_sm - 1) / a.n_sm;
        most = (int32_t)min((int64_t)0x7FFFFFFF, max((int64_t)(kPartSteps * a.hp + a.g - 1) / a.g, per));
        for (int i = threadIdx.x; i < 8 * a.n_sm; i += kListThreads) a.tickets[i] = 0;
        if (threadIdx.x == 0) s_next[0] = s_next[1] = 0;
        left = cap;
    }
    for (int64_t base = (int64_t)warp * each; base < a.S && fits; base += (int64_t)kListWarps * each) {
        if (!KEYS || !once) kept = lane < each ? packed_sequence(a, s_groups, (int32_t)min((int64_t)a.S, base + lane), bad) : PackedSequence{0, 0, 0, 0, 0};
        fits = for_items<KEYS>(a, kept, left, [&](const PackedSequence &s, int32_t i) {
            const int32_t steps = item_steps<KEYS>(a, s, i), parts = KEYS ? parts_of(steps, most) : 1;
            atomicAdd(s_bucket + bucket_of((steps + parts - 1) / parts), parts);
        });
    }
    if (!KEYS && lane == 0) s_items[warp] = fits ? (uint32_t)(cap - left) : (uint32_t)cap + 1u;
    __syncthreads();
    if (!KEYS && too_many()) return;
    static_assert(kListBuckets == kListThreads, "a thread to each bucket");
    const int32_t mine = s_bucket[threadIdx.x];
    int32_t upto = mine;
#pragma unroll
    for (int d = 1; d < kWarp; d <<= 1) {
        const int32_t o = __shfl_up_sync(kFull, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == kWarp - 1) s_warp[warp] = upto;
    __syncthreads();
    int32_t all = s_warp[lane], before = lane < warp ? all : 0;              // a lane to each warp's sum
#pragma unroll
    for (int d = kWarp / 2; d > 0; d >>= 1) {
        before += __shfl_xor_sync(kFull, before, d);
        all += __shfl_xor_sync(kFull, all, d);
    }
    s_bucket[threadIdx.x] = before + upto - mine;
    // keys: parts are at most 2 n_sm more than items, so 32 bits hold them, but they too can be more than the places where sequences overlap
    const bool full = all > cap;
    if (full) bad = true;
    if (threadIdx.x == 0) a.counts[KEYS ? 1 : 0] = full ? 0 : all;
    if (full) return;
    __syncthreads();
    left = cap;
    for (int64_t base = (int64_t)warp * each; base < a.S; base += (int64_t)kListWarps * each) {
        const PackedSequence q = once ? kept : lane < each ? packed_sequence(a, s_groups, (int32_t)min((int64_t)a.S, base + lane), bad) : PackedSequence{0, 0, 0, 0, 0};
        for_items<KEYS>(a, q, left, [&](const PackedSequence &s, int32_t i) {
            const int32_t steps = item_steps<KEYS>(a, s, i), parts = KEYS ? parts_of(steps, most) : 1, part_steps = (steps + parts - 1) / parts;
            const int32_t to = atomicAdd(s_bucket + bucket_of(part_steps), parts);
            if constexpr (KEYS) {
                const int32_t key0 = s.lo + i * kPackedRows, q0 = a.causal ? key0 : s.lo;
                int32_t slot0 = 0, ticket = 0;
                if (parts > 1) {
                    slot0 = atomicAdd(s_next, parts);
                    ticket = atomicAdd(s_next + 1, 1);
                }
                int4 *item = reinterpret_cast<int4 *>(a.key_items + to);
                for (int32_t p = 0; p < parts && HORA_IN(to + p, cap); ++p) {
                    const int64_t from = q0 + (int64_t)p * part_steps * a.tp;
                    item[2 * p] = make_int4(key0, min(kPackedRows, s.hi - key0), (int32_t)min((int64_t)s.seen_to, from),
                                            (int32_t)min((int64_t)s.seen_to, from + (int64_t)part_steps * a.tp));
                    item[2 * p + 1] = make_int4(slot0, parts, p, ticket);
                }
            } else {
                if (!HORA_IN(to, cap)) return;
                const int32_t token0 = s.lo + i * a.tile_tokens;
                int4 *item = reinterpret_cast<int4 *>(a.query_items + to);
                item[0] = make_int4(token0, min(a.tile_tokens, s.hi - token0), s.lo, s.hi);
                item[1] = make_int4(s.shared0, s.shared1, 0, 0);
            }
        });
    }
    __syncthreads();
}

// Block 0 lists the queries' items, block 1 the keys'.
__device__ __forceinline__ void packed_plan(const PackedArgs &a) {
    __shared__ int64_t s_groups[kListOffsets];
    __shared__ int32_t s_bucket[kListBuckets], s_warp[kListWarps];
    bool bad = false;
    if (a.group_offsets != nullptr) {
        for (int32_t i = threadIdx.x; i <= a.N; i += kListThreads) {
            const int64_t first = __ldcg(a.group_offsets + i);
            if (a.N < kListOffsets) s_groups[i] = first;
            if (i < a.N && __ldcg(a.group_offsets + i + 1) < first) bad = true;
        }
        if (threadIdx.x == 0 && (__ldcg(a.group_offsets) != 0 || __ldcg(a.group_offsets + a.N) + a.N != a.S)) bad = true;
    }
    if (blockIdx.x == 0 && threadIdx.x < 2) a.counts[4 + threadIdx.x] = 0;
    __syncthreads();
    // a CTA to each list
    if (blockIdx.x == 0) list_items<false>(a, s_groups, s_bucket, s_warp, bad);
    else list_items<true>(a, s_groups, s_bucket, s_warp, bad);
    if (bad) raise_status(a.status, HORA_ERR_INVALID_VALUE);
}

__global__ void __launch_bounds__(kListThreads)
packed_plan_kernel(const PackedArgs a) {
    pdl_enter();
    packed_plan(a);
}

// Of every row (token, head) lse in units of log2 and dout . out, and for fp16 the largest |dout row|^2 and |v row|^2.
template <typename T, int D>
__device__ __forceinline__ void packed_row_stats(const PackedArgs &a, int32_t cta, int32_t ctas) {
    constexpr int kLanes = D / 8, kGroups = kListThreads / kLanes, kRows = 4;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    const int32_t first = packed_offset(a, 0), tokens = max(0, packed_offset(a, a.S) - first);
    const int64_t rows = (int64_t)tokens * a.Hq, v_rows = a.half ? (int64_t)tokens * a.Hkv : 0;
    float most_d = 0.f, most_v = 0.f;
    const int64_t stride = (int64_t)ctas * kGroups;
    // a row's token and head, taken along without divisions
    const int64_t start = (int64_t)cta * kGroups + group;
    int64_t token = first + start / a.Hq;
    int32_t head = (int32_t)(start % a.Hq);
    const int32_t step_tokens = (int32_t)(stride / a.Hq), step_heads = (int32_t)(stride % a.Hq);
    for (int64_t x0 = start; __any_sync(kFull, x0 < rows); x0 += stride * kRows) {
        Raw8<T> o[kRows], d[kRows];
        int64_t at[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            zero8(o[i]);
            zero8(d[i]);
            at[i] = -1;
            if (x0 + i * stride < rows) {
                at[i] = token * a.Hq + head;
                load8(o[i], static_cast<const T *>(a.out_in) + token * a.out_stride + head * D + lane * 8);
                load8(d[i], static_cast<const T *>(a.dout) + token * a.dout_stride + head * D + lane * 8);
            }
            token += step_tokens;
            head += step_heads;
            if (head >= a.Hq) {
                head -= a.Hq;
                ++token;
            }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            float y[8], z[8], dot = 0.f, size = 0.f;
            widen8(o[i], y);
            widen8(d[i], z);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dot += y[e] * z[e];
                size += z[e] * z[e];
            }
#pragma unroll
            for (int s = kLanes / 2; s > 0; s >>= 1) dot += __shfl_xor_sync(kFull, dot, s);
            if (a.half) {
#pragma unroll
                for (int s = kLanes / 2; s > 0; s >>= 1) size += __shfl_xor_sync(kFull, size, s);
                most_d = fmaxf(most_d, size);
            }
            if (lane == 0 && at[i] >= 0) *reinterpret_cast<float2 *>(a.stats + at[i]) = make_float2(__ldcg(a.lse + at[i]) * kLog2e, dot);
        }
    }
    for (int64_t x = (int64_t)cta * kGroups + group; __any_sync(kFull, x < v_rows); x += stride) {
        Raw8<T> v;
        zero8(v);
        if (x < v_rows) load8(v, static_cast<const T *>(a.v) + (first + x / a.Hkv) * a.v_stride + x % a.Hkv * D + lane * 8);
        float z[8], size = 0.f;
        widen8(v, z);
#pragma unroll
        for (int e = 0; e < 8; ++e) size += z[e] * z[e];
#pragma unroll
        for (int s = kLanes / 2; s > 0; s >>= 1) size += __shfl_xor_sync(kFull, size, s);
        most_v = fmaxf(most_v, size);
    }
    if (a.half && lane == 0) {                           // not negative: their bits order like the numbers
        atomicMax(a.counts + 2, __float_as_int(most_d));
        atomicMax(a.counts + 3, __float_as_int(most_v));
    }
}

// The backward pass's first kernel: two CTAs for the plan, beside them the rows' statistics.
template <typename T, int D>
__global__ void __launch_bounds__(kListThreads)
packed_begin_kernel(const PackedArgs a) {
    pdl_enter();
    if (blockIdx.x < 2) packed_plan(a);
    else packed_row_stats<T, D>(a, blockIdx.x - 2, gridDim.x - 2);
}

// Heads of a tile: the most that divide g and leave no more than eight of the 128 rows idle (one head always does).
static void tile_shape(PackedArgs &a) {
    for (a.hp = a.g < kPackedRows ? a.g : kPackedRows; a.hp > 1; --a.hp)
        if (a.g % a.hp == 0 && kPackedRows / a.hp * a.hp >= kPackedRows - 8) break;
    a.tp = kPackedRows / a.hp;
    a.blocks = a.Hq / a.hp;
}

// Places of the workspace, in order; returns the bytes used.
static size_t lay_out(PackedArgs &a, bool backward, char *base) {
    size_t used = 0;
    auto take = [&](size_t bytes) {
        char *p = base + used;
        used += (bytes + 255) / 256 * 256;
        return p;
    };
    tile_shape(a);
    a.tile_tokens = backward ? a.tp : 2 * a.tp;
    a.n_sm = sm_count();
    const int64_t queries = (int64_t)a.T / a.tile_tokens + a.S, keys = (int64_t)a.T / kPackedRows + a.S + 2 * a.n_sm;
    a.query_cap = (int32_t)(queries < 0x7FFFFFFF ? queries : 0x7FFFFFFF);
    a.key_cap = (int32_t)(keys < 0x7FFFFFFF ? keys : 0x7FFFFFFF);
    a.counts = reinterpret_cast<int32_t *>(take(32));
    a.query_items = reinterpret_cast<QueryItem *>(take((size_t)a.query_cap * sizeof(QueryItem)));
    a.key_items = nullptr;
    if (backward) {
        a.key_items = reinterpret_cast<KeyItem *>(take((size_t)a.key_cap * sizeof(KeyItem)));
        a.stats = reinterpret_cast<float4 *>(take((size_t)a.T * a.Hq * sizeof(float4)));
        a.tickets = reinterpret_cast<int32_t *>(take((size_t)a.n_sm * 8 * sizeof(int32_t)));
        a.slots = reinterpret_cast<float *>(take((size_t)2 * a.n_sm * 2 * kPackedRows * a.D * sizeof(float)));
    }
    return used;
}

static bool packed_sizes(PackedArgs &a, int64_t T, int64_t S, int64_t N, int32_t Hq, int32_t Hkv, int32_t D) {
    if (T < 0 || S < 0 || N < 0 || T > 0x7FFFFF00 || S > 0x3FFFFFFF || N > S || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || Hq > 65536 || (D != 64 && D != 128)) return false;
    a.T = (int32_t)T;
    a.S = (int32_t)S;
    a.N = (int32_t)N;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.g = Hq / Hkv;
    a.D = D;
    return true;
}

static bool aligned(const void *p, uintptr_t bytes) { return !(reinterpret_cast<uintptr_t>(p) & (bytes - 1)); }

static bool packed_rows(const void *p, int64_t stride, int32_t H, int32_t D) {
    return p != nullptr && !(reinterpret_cast<uintptr_t>(p) & 15u) && stride >= (int64_t)H * D && stride % 8 == 0 && stride < (1ll << 38);
}

static hora_status_t launch_packed_plan(const PackedArgs &a, cudaStream_t stream) {
    const cudaError_t e = launch_pdl(packed_plan_kernel, 1, kListThreads, 0, stream, a);
    count_launches(1);
    return cuda_ok(e);
}

template <typename T>
static hora_status_t launch_packed_begin(const PackedArgs &a, cudaStream_t stream) {
    cudaError_t e = cudaSuccess;
    if (a.half) e = cudaMemsetAsync(a.counts + 2, 0, 8, stream);         // the largest rows so far
    const int grid = 2 + clamp_grid((int64_t)a.T * a.Hq * a.D / (kListThreads * 8 * 4) + 1, 1);
    if (e == cudaSuccess) e = a.D == 128 ? launch_pdl(packed_begin_kernel<T, 128>, grid, kListThreads, 0, stream, a) : launch_pdl(packed_begin_kernel<T, 64>, grid, kListThreads, 0, stream, a);
    count_launches(1);
    return cuda_ok(e);
}

// What both calls check and fill in alike.
static hora_status_t packed_begin(PackedArgs &a, const void *q, const void *k, const void *v, int32_t dtype, int64_t q_row_stride, int64_t k_row_stride, int64_t v_row_stride,
                                  int64_t T, const int64_t *seq_offsets, int64_t S, const int64_t *group_offsets, int64_t N, int32_t Hq, int32_t Hkv,
                                  int32_t D, float sm_scale, int32_t causal) {
    if (!packed_sizes(a, T, S, N, Hq, Hkv, D) || (dtype != HORA_DTYPE_BF16 && dtype != HORA_DTYPE_F16)) return HORA_ERR_INVALID_ARG;
    if (!(sm_scale > 0.f) || sm_scale > 1e30f || (causal != 0 && causal != 1)) return HORA_ERR_INVALID_ARG;
    if ((group_offsets == nullptr) != (N == 0)) return HORA_ERR_INVALID_ARG;
    if (T == 0 || S == 0) return HORA_OK;
    if (seq_offsets == nullptr || !aligned(seq_offsets, 8) || !aligned(group_offsets, 8) || !packed_rows(q, q_row_stride, Hq, D) || !packed_rows(k, k_row_stride, Hkv, D) || !packed_rows(v, v_row_stride, Hkv, D)) return HORA_ERR_INVALID_ARG;
    a.seq_offsets = seq_offsets;
    a.group_offsets = group_offsets;
    a.v = v;
    a.k_stride = k_row_stride;
    a.v_stride = v_row_stride;
    a.causal = causal;
    a.half = dtype == HORA_DTYPE_F16;
    a.scale = sm_scale;
    a.scale_log2 = sm_scale * kLog2e;
    return HORA_OK;
}

static hora_status_t packed_workspace(PackedArgs &a, bool backward, void *workspace, size_t bytes) {
    if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) || lay_out(a, backward, static_cast<char *>(workspace)) > bytes) return HORA_ERR_WORKSPACE;
    return HORA_OK;
}

}  // namespace hora

extern "C" size_t hora_packed_attention_workspace_bytes(int64_t T, int64_t S, int32_t Hq, int32_t Hkv, int32_t D, int32_t backward) {
    using namespace hora;
    PackedArgs a = {};
    return packed_sizes(a, T, S, 0, Hq, Hkv, D) ? lay_out(a, backward != 0, nullptr) : 0;
}

extern "C" hora_status_t hora_packed_attention(const void *q, const void *k, const void *v, int32_t dtype, int64_t q_row_stride, int64_t k_row_stride, int64_t v_row_stride,
                                               int64_t T, const int64_t *seq_offsets, int64_t S, const int64_t *group_offsets, int64_t N, int32_t Hq,
                                               int32_t Hkv, int32_t D, float sm_scale, int32_t causal, void *out, int64_t out_row_stride, float *lse,
                                               int32_t *status_dev, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace hora;
    PackedArgs a = {};
    hora_status_t rc = packed_begin(a, q, k, v, dtype, q_row_stride, k_row_stride, v_row_stride, T, seq_offsets, S, group_offsets, N, Hq, Hkv, D, sm_scale, causal);
    if (rc != HORA_OK || T == 0 || S == 0) return rc;
    if (!packed_rows(out, out_row_stride, Hq, D) || !aligned(lse, 4) || !aligned(status_dev, 4)) return HORA_ERR_INVALID_ARG;
    rc = packed_workspace(a, false, workspace, workspace_bytes);
    if (rc != HORA_OK) return rc;
    a.out = out;
    a.out_stride = out_row_stride;
    a.lse = lse;
    a.status = status_dev;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    rc = launch_packed_plan(a, s);
    return rc == HORA_OK ? launch_packed_forward(a, q, k, v, q_row_stride, dtype, s) : rc;
}

extern "C" hora_status_t hora_packed_attention_backward(const void *q, const void *k, const void *v, const void *out, const float *lse, const void *dout,
                                                        int32_t dtype, int64_t q_row_stride, int64_t k_row_stride, int64_t v_row_stride, int64_t out_row_stride,
                                                        int64_t dout_row_stride, int64_t T, const int64_t *seq_offsets, int64_t S,
                                                        const int64_t *group_offsets, int64_t N, int32_t Hq, int32_t Hkv, int32_t D, float sm_scale,
                                                        int32_t causal, void *dq, void *dk, void *dv, int64_t dq_row_stride, int64_t dk_row_stride, int64_t dv_row_stride,
                                                        int32_t *status_dev, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace hora;
    PackedArgs a = {};
    hora_status_t rc = packed_begin(a, q, k, v, dtype, q_row_stride, k_row_stride, v_row_stride, T, seq_offsets, S, group_offsets, N, Hq, Hkv, D, sm_scale, causal);
    if (rc != HORA_OK || T == 0 || S == 0) return rc;
    if (lse == nullptr || !aligned(lse, 4) || !aligned(status_dev, 4) || !packed_rows(out, out_row_stride, Hq, D) || !packed_rows(dout, dout_row_stride, Hq, D) || !packed_rows(dq, dq_row_stride, Hq, D) ||
        !packed_rows(dk, dk_row_stride, Hkv, D) || !packed_rows(dv, dv_row_stride, Hkv, D))
        return HORA_ERR_INVALID_ARG;
    rc = packed_workspace(a, true, workspace, workspace_bytes);
    if (rc != HORA_OK) return rc;
    a.out_in = out;
    a.out_stride = out_row_stride;
    a.lse = const_cast<float *>(lse);
    a.dout = dout;
    a.dout_stride = dout_row_stride;
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    a.dq_stride = dq_row_stride;
    a.dk_stride = dk_row_stride;
    a.dv_stride = dv_row_stride;
    a.status = status_dev;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    rc = dtype == HORA_DTYPE_BF16 ? launch_packed_begin<__nv_bfloat16>(a, s) : launch_packed_begin<__half>(a, s);
    return rc == HORA_OK ? launch_packed_backward(a, q, k, v, q_row_stride, dtype, s) : rc;
}
