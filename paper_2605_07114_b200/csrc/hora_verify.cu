// hora_verify_drafts: how many drafted tokens the target accepts, and the token that follows them.
//
// One thread-block cluster to a rollout.  Every CTA of it finds the first refused draft by itself (a few scalars a draft),
// which fixes the row the next token is drawn from; the CTAs then split that row's vocabulary (one does all of it
// where the rollouts fill the device).  A weight is the difference of two probabilities on the grid 2^-38, an integer, so any order of adding gives the same sum and the
// token is the one the definition names.  One pass over the row: each warp adds up segments of kSeg weights and leaves the
// sums in shared memory; the CTAs push their totals into each other's shared memory (one cluster barrier), every CTA then
// knows the drawn weight's position, and the CTA that holds it reads one segment again (from L2) to name the token.
// Bound by HBM for many rollouts (480 of 151936 fp32 values: 82 us for 455 MB; figures below are pairs from one GPU), by the chain token -> probability -> row -> barrier -> segment for few.
#include <cooperative_groups.h>

#include <utility>

#define HORA_FILE_ID 7
#include "hora_checked.cuh"
#include "hora_rows16.cuh"

HORA_CHECKED_REGISTER()

namespace hora {

namespace cg = cooperative_groups;

constexpr int kVfCluster = 8;                            // most CTAs to a rollout: the largest portable cluster
constexpr int kVfEnough = 4;                             // CTAs an SM, above which a rollout gets fewer of them
// Weights summed by one warp at a time: two (fp32: four) 16-byte loads of a lane in flight for each row, twice that for 16-bit rows
// (1920 rollouts of 50257 bf16 values: 64 -> 57 us; 480 of 151936 fp32 values would take 91 in place of 77 us).
template <typename T> constexpr int kSeg = sizeof(T) == 2 ? 1024 : 512;
constexpr int kVfMaxV = 1 << 22;

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

// A weight on the grid in two parts, hi * 2^20 + lo (lo may be negative in a difference): what a conversion to a 64-bit integer
// would give, but out of four fp32 operations.  Adding 2^23 rounding down leaves the whole part of a value below 2^23 in the
// low bits; p 2^18 minus its whole part is exact, and so is that times 2^20 before it is rounded down in turn.
struct Weight {
    int32_t hi, lo;
    __device__ __forceinline__ int64_t value() const { return ((int64_t)hi << 20) + lo; }
};
constexpr uint32_t kOneBits = 0x3F800000u;               // 1.0f: the bits of what lies outside [0, 1] (NaN, negative zero too) are larger
constexpr int32_t kWholeBits = 0x4B000000;               // 2^23

__device__ __forceinline__ Weight on_grid(float p) {     // p in [0, 1]
    const float t = __fmaf_rd(p, 262144.f, 8388608.f), rest = __fmaf_rn(p, 262144.f, 8388608.f - t), u = __fmaf_rd(rest, 1048576.f, 8388608.f);
    return {__float_as_int(t) - kWholeBits, __float_as_int(u) - kWholeBits};
}
// any p, clamped to [0, 1]; NaN and negative values count as zero and are reported in `bad`
__device__ __forceinline__ float clamped(float p, bool &bad) {
    bad |= !(p >= 0.f);
    return fminf(fmaxf(p, 0.f), 1.f);
}

__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
    return v;
}

// The rows the token is drawn from.  minus NULL: nothing to take off but, if one_hot >= 0, everything at that token.
template <typename T>
struct Rows {
    const T *plus, *minus;
    int32_t one_hot, V;

    __device__ __forceinline__ int64_t at(int32_t v, bool &bad) const {
        if (v == one_hot) return 0;
        const int64_t P = on_grid(clamped(as_float(plus[v]), bad)).value();
        const int64_t Q = minus != nullptr ? on_grid(clamped(as_float(minus[v]), bad)).value() : 0;
        return P > Q ? P - Q : 0;
    }
};

// Adds max(P - Q, 0) of eight values to the sums.
template <bool MINUS>
__device__ __forceinline__ void add8(float (&a)[8], float (&b)[8], int32_t &hi, int32_t &lo, bool &bad) {
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, MINUS ? max(__float_as_uint(a[j]), __float_as_uint(b[j])) : __float_as_uint(a[j]));
    if (most > kOneBits) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            a[j] = clamped(a[j], bad);
            if (MINUS) b[j] = clamped(b[j], bad);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        Weight w = on_grid(a[j]);
        if (MINUS) {
            const Weight q = on_grid(b[j]);
            w.hi -= q.hi;
            w.lo -= q.lo;
            if (w.hi < 0 || (w.hi == 0 && w.lo < 0)) w.hi = w.lo = 0;
        }
        hi += w.hi;
        lo += w.lo;
    }
}

// Sum of the weights of a segment's places from v0 on, for the whole warp, of a row whose 16-byte blocks begin at multiples of eight: `lead`
// elements of the first block lie before the row (element v of the row is at place v + lead).  Whole blocks are read with wide
// loads; the draft's row too where it is aligned alike (WIDE_Q).
template <typename T, bool MINUS, bool WIDE_Q>
__device__ __forceinline__ uint64_t segment_sum(const Rows<T> &r, int32_t v0, int lane, bool &bad) {
    static_assert(kSeg<T> <= 1024, "the parts of a segment's sum stay within 32 bits");
    int32_t hi = 0, lo = 0;                              // at most kSeg * 2^18 and kSeg * 2^20 over the warp
    constexpr int kSteps = kSeg<T> / (kWarp * 8);
    Raw8<T> p[kSteps], q[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int32_t v = v0 + (i * kWarp + lane) * 8;
        zero8(p[i]);
        zero8(q[i]);
        if (v >= 0 && v + 8 <= r.V) {
            load8(p[i], r.plus + v);
            if (MINUS && WIDE_Q) load8(q[i], r.minus + v);
        }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int32_t v = v0 + (i * kWarp + lane) * 8;
        float a[8], b[8];
        widen8(p[i], a);
        widen8(q[i], b);
        if (v >= 0 && v + 8 <= r.V) {
            if (MINUS && !WIDE_Q) {
#pragma unroll
                for (int j = 0; j < 8; ++j) b[j] = as_float(r.minus[v + j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (v + j >= 0 && v + j < r.V) {
                    a[j] = as_float(r.plus[v + j]);
                    if (MINUS) b[j] = as_float(r.minus[v + j]);
                }
        }
        add8<MINUS>(a, b, hi, lo, bad);
    }
    hi = __reduce_add_sync(kFull, hi);
    lo = __reduce_add_sync(kFull, lo);
    int64_t sum = ((int64_t)hi << 20) + lo;
    if (!MINUS && r.one_hot >= v0 && r.one_hot < v0 + kSeg<T> && r.one_hot >= 0 && HORA_IN(r.one_hot, r.V)) sum -= on_grid(clamped(as_float(r.plus[r.one_hot]), bad)).value();
    return (uint64_t)sum;
}

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS)
verify_kernel(const VerifyArgs a) {
    constexpr int kVfThreads = THREADS, kVfWarps = THREADS / kWarp, kSeg = hora::kSeg<T>;
    pdl_enter();
    cg::cluster_group cluster = cg::this_cluster();
    const unsigned rank = cluster.block_rank();
    const unsigned n_ctas = cluster.num_blocks();
    const int64_t r = blockIdx.x / n_ctas;
    const int lane = lane_id(), warp = threadIdx.x >> 5;
    extern __shared__ uint64_t s_seg[];                  // [segs_per_cta]
    __shared__ uint64_t s_total[2][kVfCluster];          // pushed by every CTA of the cluster, one row for each attempt
    __shared__ uint64_t s_warp[kVfWarps];
    __shared__ int32_t s_n, s_len, s_pick;
    __shared__ uint64_t s_before;
    bool bad = false;
    auto begun = cluster.barrier_arrive();               // shared memory of the others may be written once all have begun

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
    // a token outside the vocabulary was refused for that: the row has no place for it, and nothing is taken off
    const int32_t refused = (n < len && a.draft == nullptr) ? __ldcg(a.draft_tokens + r * a.K + n) : -1;
    rows.one_hot = refused < a.V ? refused : -1;

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
            const uint64_t w = rows.minus == nullptr ? segment_sum<T, false, true>(rows, v0, lane, bad)
                               : wide_q ? segment_sum<T, true, true>(rows, v0, lane, bad) : segment_sum<T, true, false>(rows, v0, lane, bad);
            if (lane == 0) s_seg[s] = w;
        }
        __syncthreads();
        if (attempt == 0) cluster.barrier_wait(std::move(begun));
        if (warp == 0) {
            uint64_t w = 0;
            for (int32_t s = lane; s < n_segs; s += kWarp) w += s_seg[s];
            w = warp_sum(w);
            if (lane < n_ctas) *cluster.map_shared_rank(&s_total[attempt][rank], lane) = w;
        }
        cluster.sync();
        total = 0;
        for (unsigned c = 0; c < n_ctas; ++c) {
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
        w[j] = (v0 + j >= 0 && v0 + j < a.V) ? (uint64_t)rows.at(v0 + j, ignore) : 0;
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
    const int32_t seg = es == 2 ? kSeg<__half> : kSeg<float>, segs = (V + 16 / es - 1 + seg - 1) / seg;
    // Many CTAs to a rollout while that fills the device, fewer where the rollouts do it by themselves: the chain before and after the
    // pass over the row costs every CTA the same (1920 rollouts of 50257 16-bit values: 173 us with eight, 72 with one).
    int ctas = kVfCluster;
    while (ctas > 1 && R * (ctas / 2) >= (int64_t)sm_count() * kVfEnough && (segs + ctas / 2 - 1) / (ctas / 2) <= 4096) ctas /= 2;
    a.segs_per_cta = (segs + ctas - 1) / ctas;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(R * ctas));
    // eight warps to a CTA where its latency counts, four where it is one of many (480 rollouts: 81 -> 77 us; 8 rollouts: 18 us with four, 13 with eight)
    const int threads = ctas == kVfCluster ? 256 : 128;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)a.segs_per_cta * 8;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    auto go = [&](auto few, auto many) { return cudaLaunchKernelEx(&cfg, threads == 256 ? few : many, a); };
    cudaError_t e;
    if (dtype == HORA_DTYPE_F32) e = go(verify_kernel<float, 256>, verify_kernel<float, 128>);
    else if (dtype == HORA_DTYPE_BF16) e = go(verify_kernel<__nv_bfloat16, 256>, verify_kernel<__nv_bfloat16, 128>);
    else e = go(verify_kernel<__half, 256>, verify_kernel<__half, 128>);
    count_launches(1);
    return cuda_ok(e);
}
