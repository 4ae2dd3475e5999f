// hora_packed_attention: the forward kernel.
//
// Per row: m the running maximum of s = scale q.k (in units of log2), l = sum 2^(s - m), o = sum 2^(s - m) v;  out = o / l,
// lse = m ln 2 + log l.  A CTA holds an SM and works on two tiles of 128 query rows at a time, which share the keys and values:
// while the softmax of one is under way the tensor cores do the products of the other.  Four warps do a tile's softmax, one thread to a row;
// one warp brings in queries, keys and values by TMA, one issues the products.  S = Q K^T (128 x 128) is accumulated in tensor memory, the
// weights P replace it there in 16 bits (rounded once, as the product needs them; sums are of the unrounded ones) and are the left
// operand of O += P V.
//   The products of a tile complete in the order in which they are issued, so when S of a step has arrived, O holds all steps before, and may
// be scaled: which is done only when a row's maximum has grown by more than 2^8 (weights up to 256 are as exact as weights up to 1).
//   Keys that are not of the sequence are in no row's sum; the product stops at the last sixteen that hold one of it, and values
// of others among those are cleared in shared memory first, since 0 * NaN is not 0.
//   Every wait has a limit; a wait that reaches it makes the CTA give up and report HORA_ERR_INTERNAL.
#define HORA_FILE_ID 11
#include <type_traits>

#include "hora_packed_attention.cuh"

HORA_CHECKED_REGISTER()

namespace hora {

namespace {

constexpr int kTile = kPackedRows;
constexpr int kLoadWarp = 8, kProductWarp = 9;

template <int D>
struct ForwardSmem {
    static constexpr int kTileBytes = kTile * D * 2;
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int kQ = 0, kRing = 2 * kTileBytes, kSmall = kRing + kStages * kTileBytes;
};

struct ForwardShared {
    uint64_t full[10], empty[10], queries, queries_free, scores[2], weights[2], output[2], output_free[2];
    int32_t failed;
    uint32_t tmem;
};

// An item as the warps need it: runs of keys, steps of each tile.
struct Item {
    int32_t token0, end, own0, shared0, shared1, last_token;
    int32_t block;
    int32_t n_shared, n[2], tokens[2];
    bool valid;

    __device__ __forceinline__ int32_t steps() const { return max(n[0], n[1]); }
    // first key of step j and how many keys of the sequence there are from it on
    __device__ __forceinline__ void keys(int32_t j, int32_t &key0, int32_t &count) const {
        if (j < n_shared) {
            key0 = shared0 + j * kTile;
            count = shared1 - key0;
        } else {
            key0 = own0 + (j - n_shared) * kTile;
            count = end - key0;
        }
        count = min(count, kTile);
    }
};

struct RawItem {
    int4 a, b;
    int32_t block;
    bool valid;
};

__device__ __forceinline__ RawItem fetch_item(const PackedArgs &a, int32_t r, int32_t n_items) {
    const int64_t x = dealt(r);
    RawItem f = {};
    f.valid = x < (int64_t)n_items * a.blocks;
    if (!f.valid) return f;
    const int64_t i = x / a.blocks;
    f.block = (int32_t)(x - i * a.blocks);
    const int4 *p = reinterpret_cast<const int4 *>(a.query_items + i);
    f.a = __ldcg(p);
    f.b = __ldcg(p + 1);
    return f;
}

__device__ __forceinline__ Item make_item(const PackedArgs &a, const RawItem &f) {
    Item q;
    q.valid = f.valid;
    q.token0 = f.a.x;
    q.own0 = f.a.z;
    q.end = f.a.w;
    q.shared0 = f.b.x;
    q.shared1 = f.b.y;
    q.block = f.block;
    q.n_shared = (q.shared1 - q.shared0 + kTile - 1) / kTile;
    q.tokens[0] = min(a.tp, f.a.y);
    q.tokens[1] = f.a.y - q.tokens[0];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int32_t last = a.causal ? q.token0 + t * a.tp + q.tokens[t] : q.end;
        q.n[t] = q.tokens[t] > 0 ? q.n_shared + (last - q.own0 + kTile - 1) / kTile : 0;
    }
    return q;
}

extern __shared__ __align__(1024) uint8_t s_forward[];

template <typename Q, int D>
__global__ void __launch_bounds__(kPackedThreads, 1)
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
                   scores = smem_at(sh.scores), weights = smem_at(sh.weights), output = smem_at(sh.output), output_free = smem_at(sh.output_free);
    if (threadIdx.x == 0) {
        sh.failed = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(full + 8 * s, 1);
            bar_init(empty + 8 * s, 1);
        }
        bar_init(queries, 1);
        bar_init(queries_free, 1);
        for (int t = 0; t < 2; ++t) {
            bar_init(scores + 8 * t, 1);
            bar_init(weights + 8 * t, kTile);
            bar_init(output + 8 * t, 1);
            bar_init(output_free + 8 * t, kTile);
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
    const int32_t n_items = __ldcg(a.counts);
    bool ok = true;

    if (warp == kLoadWarp) {
        if (lane == 0) {
            int32_t pos = 0;                             // copies into the ring so far
            uint32_t turn = 0;
            RawItem next = fetch_item(a, 0, n_items);
            for (int32_t r = 0; next.valid && ok; ++r, ++turn) {
                const Item it = make_item(a, next);
                next = fetch_item(a, r + 1, n_items);
                const int32_t head = it.block * a.hp / a.g;
                const int tiles = it.tokens[1] > 0 ? 2 : 1;
                if (r > 0) ok = bar_wait(queries_free, (turn + 1) & 1, failed);
                if (!ok) break;
                bar_expect(queries, tiles * kParts * a.hp * a.tp * 128);
                for (int t = 0; t < tiles; ++t)
                    for (int p = 0; p < kParts; ++p)
                        tma_box3(base + Smem::kQ + t * Smem::kTileBytes + p * (kTile * 128), &q_map, p * 64, it.block * a.hp, it.token0 + t * a.tp, queries);
                const int32_t n = it.steps();
                for (int32_t j = 0; j < n && ok; ++j) {
                    int32_t key0, count;
                    it.keys(j, key0, count);
                    for (int which = 0; which < 2 && ok; ++which, ++pos) {
                        const int stage = pos % kStages;
                        if (pos >= kStages) ok = bar_wait(empty + 8 * stage, (pos / kStages + 1) & 1, failed);
                        if (!ok) break;
                        bar_expect(full + 8 * stage, Smem::kTileBytes);
                        for (int p = 0; p < kParts; ++p)
                            tma_box3(base + Smem::kRing + stage * Smem::kTileBytes + p * (kTile * 128), which ? &v_map : &k_map, p * 64, head, key0, full + 8 * stage);
                    }
                }
            }
            // the CTA may not end while copies are on their way to it: each is waited for by its use, unless the CTA has given up
            if (!ok) {
                int32_t never = 0;
                for (int32_t x = max(0, pos - kStages); x < pos; ++x) bar_wait(full + 8 * (x % kStages), (x / kStages) & 1, &never);
                if (turn > 0) bar_wait(queries, (turn - 1) & 1, &never);
            }
        }
    } else if (warp == kProductWarp) {
        constexpr uint32_t kType = std::is_same<Q, __nv_bfloat16>::value ? 1u : 0u;
        constexpr uint32_t kIdescS = (1u << 4) | (kType << 7) | (kType << 10) | ((kTile / 8) << 17) | ((kTile / 16) << 24);
        constexpr uint32_t kIdescO = (1u << 4) | (kType << 7) | (kType << 10) | (1u << 16) | ((D / 8) << 17) | ((kTile / 16) << 24);
        const uint32_t k0 = operand(base + Smem::kRing, 16), v0 = operand(base + Smem::kRing, kTile * 128), q0 = operand(base + Smem::kQ, 16);
        uint32_t weights_phase = 0, free_phase = 0, started = 0;
        int32_t pos = 0;
        RawItem next = fetch_item(a, 0, n_items);
        for (int32_t r = 0; next.valid && ok; ++r) {
            const Item it = make_item(a, next);
            next = fetch_item(a, r + 1, n_items);
            const int32_t n = it.steps();
            auto stage_of = [&](int32_t j, int which) { return (uint32_t)((pos + 2 * j + which) % kStages); };
            auto arrived = [&](int32_t j, int which) {
                const int32_t x = pos + 2 * j + which;
                return bar_wait(full + 8 * (x % kStages), (x / kStages) & 1, failed);
            };
            auto scores_of = [&](int t, int32_t j) {
                if (elect_one()) {
                    const uint32_t k = k0 + stage_of(j, 0) * (Smem::kTileBytes >> 4), q = q0 + t * (Smem::kTileBytes >> 4);
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) {
                        const uint32_t off = ((x >> 2) * (kTile * 128) + (x & 3) * 32) >> 4;
                        mma_smem(tmem + t * kTile, q + off, k + off, kIdescS, x > 0);
                    }
                    mma_commit(scores + 8 * t);
                }
                __syncwarp();
            };
            ok = bar_wait(queries, r & 1, failed) && arrived(0, 0);
            if (!ok) break;
            fence_after();
            for (int t = 0; t < 2; ++t)
                if (it.n[t] > 0) scores_of(t, 0);
            if (elect_one()) {
                mma_commit(empty + 8 * stage_of(0, 0));
                if (n == 1) mma_commit(queries_free);
            }
            __syncwarp();
            for (int32_t j = 0; j < n && ok; ++j) {
                int32_t key0, count;
                it.keys(j, key0, count);
                ok = arrived(j, 1);
                if (!ok) break;
                if (count & 15) {                        // values that are not of the sequence, among the last sixteen
                    const uint32_t at = base + Smem::kRing + stage_of(j, 1) * Smem::kTileBytes;
                    const int32_t clear = ((count + 15) & ~15) - count;
                    for (int32_t c = lane; c < clear * (D / 8); c += kWarp) {
                        const uint32_t to = at + (c % (D / 8) >> 3) * (kTile * 128) + (count + c / (D / 8)) * 128 + (c & 7) * 16;
                        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(to), "r"(0) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                for (int t = 0; t < 2 && ok; ++t) {
                    if (j < it.n[t]) {
                        ok = bar_wait(weights + 8 * t, (weights_phase >> t) & 1, failed);
                        weights_phase ^= 1u << t;
                        if (ok && j == 0 && ((started >> t) & 1)) {      // the output of the item before has been read
                            ok = bar_wait(output_free + 8 * t, (free_phase >> t) & 1, failed);
                            free_phase ^= 1u << t;
                        }
                        if (!ok) break;
                        started |= 1u << t;
                        fence_after();
                        if (elect_one()) {
                            const uint32_t v = v0 + stage_of(j, 1) * (Smem::kTileBytes >> 4), w = tmem + t * kTile;
#pragma unroll
                            for (int g = 0; g < kTile / 16; ++g)
                                if (g * 16 < count) mma_tmem(tmem + 256 + t * D, w + g * 8, v + g * (2048 >> 4), kIdescO, j > 0 || g > 0);
                            if (j == it.n[t] - 1) mma_commit(output + 8 * t);
                        }
                        __syncwarp();
                    }
                    if (j + 1 < it.n[t]) {
                        ok = arrived(j + 1, 0);
                        if (!ok) break;
                        fence_after();
                        scores_of(t, j + 1);
                    }
                }
                if (!ok) break;
                if (elect_one()) {
                    mma_commit(empty + 8 * stage_of(j, 1));
                    if (j + 1 < n) mma_commit(empty + 8 * stage_of(j + 1, 0));
                    if (j + 2 == n) mma_commit(queries_free);
                }
                __syncwarp();
            }
            pos += 2 * n;
        }
    } else if (warp < 8) {
        // ---- softmax: thread `row` of a tile has row `row` of its scores
        const int t = warp >> 2, row = threadIdx.x & (kTile - 1);
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
        const uint32_t t_s = lanes + t * kTile, t_o = lanes + 256 + t * D;
        const int32_t row_token = row / a.hp, row_head = row - row_token * a.hp;
        uint32_t scores_phase = 0, n_output = 0;
        RawItem next = fetch_item(a, 0, n_items);
        for (int32_t r = 0; next.valid && ok; ++r) {
            const Item it = make_item(a, next);
            next = fetch_item(a, r + 1, n_items);
            const int32_t n = it.n[t];
            if (n == 0) continue;
            const int32_t token = it.token0 + t * a.tp + row_token;
            const bool have = row_token < it.tokens[t];
            const int32_t seen_to = a.causal && have ? min(it.end, token + 1) : it.end;
            float m = -INFINITY, l = 0.f;
            for (int32_t j = 0; j < n; ++j) {
                int32_t limit;                           // keys of the step that the row sees
                if (j < it.n_shared) limit = it.shared1 - it.shared0 - j * kTile;
                else limit = seen_to - it.own0 - (j - it.n_shared) * kTile;
                ok = bar_wait(scores + 8 * t, scores_phase, failed);
                scores_phase ^= 1;
                ok = __all_sync(kFull, ok);
                if (!ok) break;
                fence_after();
                float s[4][32];
#pragma unroll
                for (int b = 0; b < 4; ++b) tmem_load(t_s + b * 32, s[b]);
                tmem_load_wait();
                if (__any_sync(kFull, limit < kTile)) {
#pragma unroll
                    for (int b = 0; b < 4; ++b)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (b * 32 + e >= limit) s[b][e] = -INFINITY;
                }
                float t4[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    t4[b] = s[b][0];
#pragma unroll
                    for (int e = 1; e < 31; e += 2) t4[b] = fmaxf(t4[b], fmaxf(s[b][e], s[b][e + 1]));
                    t4[b] = fmaxf(t4[b], s[b][31]);
                }
                const float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])) * a.scale_log2;
                if (j == 0) {
                    m = top;
                } else if (__any_sync(kFull, have && top > m + 8.f)) {      // rows of no token may hold anything: they have no say
                    const float up = fmaxf(m, top), f = up == -INFINITY ? 1.f : exp2_approx(m - up);
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
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int b = 0; b < 8; ++b) {
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float2 y = make_float2(s[b >> 1][(b & 1) * 16 + 2 * e], s[b >> 1][(b & 1) * 16 + 2 * e + 1]);
                        y = fma2(y, make_float2(a.scale_log2, a.scale_log2), make_float2(-z, -z));
                        y = make_float2(exp2_approx(y.x), exp2_approx(y.y));
                        sum = add2(sum, y);
                        w[e] = pack2(y.x, y.y, Q());
                    }
                    tmem_store8(t_s + b * 8, w);
                }
                l += sum.x + sum.y;
                tmem_store_wait();
                fence_before();
                bar_arrive(weights + 8 * t);
            }
            if (!ok) break;
            ok = bar_wait(output + 8 * t, n_output++ & 1, failed);
            ok = __all_sync(kFull, ok);
            if (!ok) break;
            fence_after();
            const float inv = l == 0.f ? 0.f : 1.f / l;       // NaN where a score was NaN: it is in no maximum, but in the sum
            const int32_t head = it.block * a.hp + row_head;
            Q *out = static_cast<Q *>(a.out) + (int64_t)token * a.out_stride + (int64_t)head * D;
#pragma unroll 1
            for (int b = 0; b < D / 32; ++b) {
                float o[32];
                tmem_load(t_o + b * 32, o);
                tmem_load_wait();
                if (have) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = o[v * 8 + e] * inv;
                        *reinterpret_cast<uint4 *>(out + b * 32 + v * 8) = pack8<Q>(x);
                    }
                }
            }
            fence_before();
            bar_arrive(output_free + 8 * t);
            if (have && a.lse != nullptr) a.lse[(int64_t)token * a.Hq + head] = (m == -INFINITY ? 0.f : kLn2 * m) + logf(l);
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
    if (!head_map(&q_map, q, dtype, D, a.Hq, a.T, q_stride, a.hp, a.tp) || !head_map(&k_map, k, dtype, D, a.Hkv, a.T, a.kv_stride, 1, kTile) ||
        !head_map(&v_map, v, dtype, D, a.Hkv, a.T, a.kv_stride, 1, kTile))
        return HORA_ERR_CUDA;
    constexpr int kSmem = ForwardSmem<D>::kSmall + (int)sizeof(ForwardShared);
    static std::atomic<uint64_t> devices{0};
    cudaError_t e = allow_shared(reinterpret_cast<const void *>(packed_forward_kernel<Q, D>), kSmem, devices);
    const int64_t most = (int64_t)a.query_cap * a.blocks;
    if (e == cudaSuccess) e = launch_pdl(packed_forward_kernel<Q, D>, clamp_grid(most, 1), kPackedThreads, kSmem, stream, a, q_map, k_map, v_map);
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
