// hora_verify_drafts: how many drafted tokens the target accepts, and the token that follows them.
//
// One thread-block cluster to a rollout.  Every CTA of it finds the first refused draft by itself (a few scalars a draft),
// which fixes the row the next token is drawn from; the CTAs then split that row's vocabulary.  A weight is the
// difference of two probabilities on the grid 2^-38, an integer, so any order of adding gives the same sum and the
// token is the one the definition names.  One pass over the row: each warp adds up segments of kSeg weights and leaves the
// sums in shared memory; the CTAs push their totals into each other's shared memory (one cluster barrier), every CTA then
// knows the drawn weight's position, and the CTA that holds it reads one segment again (from L2) to name the token.
// Bound by HBM for many rollouts, by the chain token -> probability -> row -> barrier -> segment for few.
#include <cooperative_groups.h>

#include "hora_rows16.cuh"

namespace hora {

namespace cg = cooperative_groups;

constexpr int kVfThreads = 256;
constexpr int kVfWarps = kVfThreads / kWarp;
constexpr int kVfCluster = 8;                            // CTAs to a rollout: the largest portable cluster
constexpr int kSeg = 512;                                // weights summed by one warp at a time
constexpr int kVfMaxV = 1 << 22;
constexpr int kMaxSegs = kVfMaxV / kVfCluster / kSeg + 1;  // segments of one CTA (a row may begin inside a block)
constexpr float kGrid = 274877906944.f;                  // 2^38

struct VerifyArgs {
    const void *target, *draft;
    int64_t target_stride, draft_stride;
    const int32_t *draft_tokens, *draft_len;
    const float *u_accept, *u_sample;
    int32_t *n_accepted, *tokens, *status;
    int32_t K, V, segs_per_cta;
};

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }

// p on the grid, in [0, 2^38]; NaN and negative values count as zero and are reported in `bad`
__device__ __forceinline__ uint64_t grid_weight(float p, bool &bad) {
    bad |= !(p >= 0.f);
    return (uint64_t)(fminf(fmaxf(p, 0.f), 1.f) * kGrid);
}

__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
    return v;
}

// The rows the token is drawn from.  minus_row NULL: nothing to take off but, if one_hot >= 0, everything at that token.
template <typename T>
struct Rows {
    const T *plus, *minus;
    int32_t one_hot, V;

    __device__ __forceinline__ uint64_t weight(float p, float q, int32_t v, bool &bad) const {
        const uint64_t P = grid_weight(p, bad);
        uint64_t Q = minus != nullptr ? grid_weight(q, bad) : 0;
        if (v == one_hot) Q = (uint64_t)kGrid;
        return P > Q ? P - Q : 0;
    }
    __device__ __forceinline__ uint64_t at(int32_t v, bool &bad) const {
        return weight(as_float(plus[v]), minus != nullptr ? as_float(minus[v]) : 0.f, v, bad);
    }
};

// Sum of the weights [v0, v0 + kSeg) of a row whose 16-byte blocks begin at multiples of eight: `lead` elements of
// the first block lie before the row (element v of the row is at place v + lead).  Whole blocks are read with wide
// loads; the draft's row too where it is aligned alike (WIDE_Q).
template <typename T, bool WIDE_Q>
__device__ __forceinline__ uint64_t segment_sum(const Rows<T> &r, int32_t v0, int lane, bool &bad) {
    uint64_t sum = 0;
    constexpr int kSteps = kSeg / (kWarp * 8);
    Raw8<T> p[kSteps], q[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int32_t v = v0 + (i * kWarp + lane) * 8;
        zero8(p[i]);
        zero8(q[i]);
        if (v >= 0 && v + 8 <= r.V) {
            load8(p[i], r.plus + v);
            if (WIDE_Q && r.minus != nullptr) load8(q[i], r.minus + v);
        }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int32_t v = v0 + (i * kWarp + lane) * 8;
        if (v >= 0 && v + 8 <= r.V) {
            float a[8], b[8];
            widen8(p[i], a);
            widen8(q[i], b);
            if (!WIDE_Q && r.minus != nullptr) {
#pragma unroll
                for (int j = 0; j < 8; ++j) b[j] = as_float(r.minus[v + j]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += r.weight(a[j], b[j], v + j, bad);
        } else {
            for (int j = 0; j < 8; ++j)
                if (v + j >= 0 && v + j < r.V) sum += r.at(v + j, bad);
        }
    }
    return sum;
}

template <typename T>
__global__ void __cluster_dims__(kVfCluster, 1, 1) __launch_bounds__(kVfThreads)
verify_kernel(const VerifyArgs a) {
    pdl_enter();
    cg::cluster_group cluster = cg::this_cluster();
    const unsigned rank = cluster.block_rank();
    const int64_t r = blockIdx.x / kVfCluster;
    const int lane = lane_id(), warp = threadIdx.x >> 5;
    __shared__ uint64_t s_seg[kMaxSegs];
    __shared__ uint64_t s_total[2][kVfCluster];          // pushed by every CTA of the cluster, one row for each attempt
    __shared__ uint64_t s_warp[kVfWarps];
    __shared__ int32_t s_n, s_len, s_pick;
    __shared__ uint64_t s_before;
    bool bad = false;

    if (warp == 0) {
        int32_t len = a.draft_len ? __ldcg(a.draft_len + r) : a.K;
        if (len < 0 || len > a.K) { bad = true; len = len < 0 ? 0 : a.K; }
        int32_t n = len;
        for (int32_t base = 0; base < len; base += kWarp) {
            const int32_t t = base + lane;
            bool refuse = false;
            if (t < len) {
                const int32_t x = __ldcg(a.draft_tokens + r * a.K + t);
                refuse = x < 0 || x >= a.V;
                bad |= refuse;
                if (!refuse) {
                    const double p = as_float(static_cast<const T *>(a.target)[(r * (a.K + 1) + t) * a.target_stride + x]);
                    const double q = a.draft ? as_float(static_cast<const T *>(a.draft)[(r * a.K + t) * a.draft_stride + x]) : 1.f;
                    refuse = !((double)__ldcg(a.u_accept + r * a.K + t) * q < p);      // exact: two 24-bit factors
                }
            }
            const unsigned ballot = __ballot_sync(kFull, refuse);
            if (ballot) { n = base + __ffs(ballot) - 1; break; }
        }
        if (lane == 0) { s_n = n; s_len = len; }
    }
    __syncthreads();
    const int32_t n = s_n, len = s_len;
    Rows<T> rows;
    rows.V = a.V;
    rows.plus = static_cast<const T *>(a.target) + (r * (a.K + 1) + n) * a.target_stride;
    rows.minus = (n < len && a.draft != nullptr) ? static_cast<const T *>(a.draft) + (r * a.K + n) * a.draft_stride : nullptr;
    rows.one_hot = (n < len && a.draft == nullptr) ? __ldcg(a.draft_tokens + r * a.K + n) : -1;

    // the vocabulary in blocks of 16 bytes as they lie in memory: `lead` elements of the first one are not the row's
    constexpr int kPer16 = 16 / sizeof(T);
    const int32_t lead = (int32_t)((reinterpret_cast<uintptr_t>(rows.plus) & 15u) / sizeof(T));
    const bool wide_q = rows.minus == nullptr ||
                        ((reinterpret_cast<uintptr_t>(rows.minus) ^ reinterpret_cast<uintptr_t>(rows.plus)) & 15u) == 0;
    static_assert(8 % kPer16 == 0, "a lane's eight elements are whole blocks");
    const int32_t seg0 = (int32_t)rank * a.segs_per_cta;
    const int32_t all_segs = (a.V + lead + kSeg - 1) / kSeg;
    const int32_t n_segs = min(a.segs_per_cta, max(0, all_segs - seg0));

    uint64_t total = 0, mine = 0, first = 0;
    for (int attempt = 0; attempt < 2; ++attempt) {
        for (int32_t s = warp; s < n_segs; s += kVfWarps) {
            const int32_t v0 = (seg0 + s) * kSeg - lead;
            const uint64_t w = warp_sum(wide_q ? segment_sum<T, true>(rows, v0, lane, bad) : segment_sum<T, false>(rows, v0, lane, bad));
            if (lane == 0) s_seg[s] = w;
        }
        __syncthreads();
        if (warp == 0) {
            uint64_t w = 0;
            for (int32_t s = lane; s < n_segs; s += kWarp) w += s_seg[s];
            w = warp_sum(w);
            if (attempt == 0) cluster.barrier_wait(cluster.barrier_arrive());
            if (lane < kVfCluster) *cluster.map_shared_rank(&s_total[attempt][rank], lane) = w;
        } else if (attempt == 0) {
            cluster.barrier_wait(cluster.barrier_arrive());
        }
        cluster.sync();
        total = 0;
        for (unsigned c = 0; c < kVfCluster; ++c) {
            const uint64_t w = s_total[attempt][c];
            if (c < rank) first += w;
            if (c == rank) mine = w;
            total += w;
        }
        if (total != 0 || (rows.minus == nullptr && rows.one_hot < 0)) break;
        rows.minus = nullptr;                            // nothing is left of the difference: draw from the target itself
        rows.one_hot = -1;
        first = 0;
    }
    if (bad) raise_status(a.status, HORA_ERR_INVALID_VALUE);

    int32_t *__restrict__ out = a.tokens + r * (a.K + 1);
    if (rank == 0) {
        if (threadIdx.x == 0) a.n_accepted[r] = n;
        for (int32_t t = threadIdx.x; t <= a.K; t += kVfThreads)
            if (t != n) out[t] = t < n ? __ldcg(a.draft_tokens + r * a.K + t) : -1;
    }
    if (total == 0) {
        if (rank == 0 && threadIdx.x == 0) {
            out[n] = -1;
            raise_status(a.status, HORA_ERR_INVALID_VALUE);
        }
        return;
    }
    // floor(U * total) with U = k 2^-24: the product has at most 60 + 24 bits
    const float u = __ldcg(a.u_sample + r);
    const uint64_t k = (uint64_t)fminf(fmaxf(u * 16777216.f, 0.f), 16777215.f);
    const uint64_t limit = (__umul64hi(total, k) << 40) | ((total * k) >> 24);
    if (limit < first || limit >= first + mine) return;  // uniform over the CTA: another one holds the token

    // the segment that holds weight number `limit`, by one warp over the segment sums
    if (warp == 0) {
        uint64_t before = first;
        for (int32_t base = 0; base < n_segs; base += kWarp) {
            const uint64_t w = base + lane < n_segs ? s_seg[base + lane] : 0;
            uint64_t incl = w;
#pragma unroll
            for (int d = 1; d < kWarp; d <<= 1) {
                const uint64_t o = __shfl_up_sync(kFull, incl, d);
                if (lane >= d) incl += o;
            }
            const unsigned hit = __ballot_sync(kFull, before + incl > limit);
            if (hit) {
                const int src = __ffs(hit) - 1;
                before += __shfl_sync(kFull, incl - w, src);
                if (lane == 0) { s_pick = base + src; s_before = before; }
                break;
            }
            before += __shfl_sync(kFull, incl, kWarp - 1);
        }
    }
    __syncthreads();
    // that segment again, kSeg / kVfThreads neighbouring weights a thread
    constexpr int kEach = kSeg / kVfThreads;
    const int32_t v0 = (seg0 + s_pick) * kSeg - lead + threadIdx.x * kEach;
    uint64_t w[kEach], incl = 0;
    bool ignore = false;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        w[j] = (v0 + j >= 0 && v0 + j < a.V) ? rows.at(v0 + j, ignore) : 0;
        incl += w[j];
    }
    const uint64_t own = incl;
#pragma unroll
    for (int d = 1; d < kWarp; d <<= 1) {
        const uint64_t o = __shfl_up_sync(kFull, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == kWarp - 1) s_warp[warp] = incl;
    __syncthreads();
    uint64_t run = s_before + incl - own;
    for (int i = 0; i < warp; ++i) run += s_warp[i];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if (run <= limit && limit < run + w[j]) out[n] = v0 + j;
        run += w[j];
    }
}

}  // namespace hora

extern "C" hora_status_t hora_verify_drafts(const void *target, int32_t dtype, int64_t target_row_stride, const void *draft,
                                            int64_t draft_row_stride, const int32_t *draft_tokens, const int32_t *draft_len,
                                            int64_t R, int32_t K, int32_t V, const float *u_accept, const float *u_sample,
                                            int32_t *n_accepted, int32_t *tokens, int32_t *status_dev, void *stream) {
    using namespace hora;
    const int es = dtype == HORA_DTYPE_E4M3 ? 0 : dtype_bytes(dtype);
    if (es == 0 || R < 0 || R > 0x7FFFFFFF / kVfCluster || K < 0 || K > 255 || V < 1 || V > kVfMaxV) return HORA_ERR_INVALID_ARG;
    if (R == 0) return HORA_OK;
    if (target == nullptr || u_sample == nullptr || n_accepted == nullptr || tokens == nullptr) return HORA_ERR_INVALID_ARG;
    if (target_row_stride < V || (reinterpret_cast<uintptr_t>(target) % es) != 0) return HORA_ERR_INVALID_ARG;
    if (K > 0 && (draft_tokens == nullptr || u_accept == nullptr)) return HORA_ERR_INVALID_ARG;
    if (K > 0 && draft != nullptr && (draft_row_stride < V || (reinterpret_cast<uintptr_t>(draft) % es) != 0)) return HORA_ERR_INVALID_ARG;
    VerifyArgs a;
    a.target = target;
    a.draft = K > 0 ? draft : nullptr;
    a.target_stride = target_row_stride;
    a.draft_stride = draft_row_stride;
    a.draft_tokens = draft_tokens;
    a.draft_len = K > 0 ? draft_len : nullptr;
    a.u_accept = u_accept;
    a.u_sample = u_sample;
    a.n_accepted = n_accepted;
    a.tokens = tokens;
    a.status = status_dev;
    a.K = K;
    a.V = V;
    // the most segments a row can have, with up to a block's worth of elements in front of it
    const int32_t segs = (V + 16 / es - 1 + kSeg - 1) / kSeg;
    a.segs_per_cta = (segs + kVfCluster - 1) / kVfCluster;
    const int grid = (int)(R * kVfCluster);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (dtype == HORA_DTYPE_F32) e = launch_pdl(verify_kernel<float>, grid, kVfThreads, 0, s, a);
    else if (dtype == HORA_DTYPE_BF16) e = launch_pdl(verify_kernel<__nv_bfloat16>, grid, kVfThreads, 0, s, a);
    else e = launch_pdl(verify_kernel<__half>, grid, kVfThreads, 0, s, a);
    count_launches(1);
    return cuda_ok(e);
}
