// hora_group_attention: plan, joining of the partial results, and the C entry.
#define HORA_FILE_ID 5
#include "hora_group_attention.cuh"

HORA_CHECKED_REGISTER()

namespace hora {

constexpr int kPlanThreads = 1024;
constexpr int kPlanKept = 4;                             // sequences of a thread whose steps it keeps in registers
constexpr int kPlanOffsets = 4096;                       // group offsets kept in shared memory for the searches
// The wide items' pass costs about 15 us however little there is to do in it: they are taken as narrow ones instead while
// that makes no more than this many steps a stream (of 8 rows and 16 or 32 keys, about a microsecond each).
#ifdef HORA_CHECKED
constexpr int kWideWorth = -1;                           // the checked build takes the wide way wherever it can: small problems check it too
#else
constexpr int kWideWorth = 16;
#endif

// start[line][i] = steps before sequence i on its line, group_of[r].  One CTA: every thread takes a run of sequences.
__global__ void __launch_bounds__(kPlanThreads)
attention_plan_kernel(const AttnArgs a) {
    pdl_enter();
    __shared__ int64_t s_warp[3][kPlanThreads / kWarp];
    static_assert(kPlanThreads / kWarp == kWarp, "a lane to each warp's sums");
    __shared__ int64_t s_off[kPlanOffsets];
    const int64_t n = (int64_t)a.N + a.R;
    const int64_t each = (n + kPlanThreads - 1) / kPlanThreads;
    const int64_t lo = min(n, each * threadIdx.x), hi = min(n, lo + each);
    bool bad = false, ignore = false;
    // steps of the sequences that are narrow anyhow; of those that can be wide, as wide and as narrow ones
    enum { kNarrow, kWide, kEither, kSums };
    int64_t sum[kSums] = {0, 0, 0}, run[kSums], all[kSums];
    // of this thread's first sequences: steps as wide ones (0: always narrow), as narrow ones.  One sequence can have more than 2^31 of them
    // (a million one-byte keys under 2100 rollouts with 32 cache heads).
    int64_t kept[kPlanKept][2];
    const bool in_shared = a.N + 1 <= kPlanOffsets;
    if (in_shared)
        for (int32_t i = threadIdx.x; i <= a.N; i += kPlanThreads) s_off[i] = __ldcg(a.group_offsets + i);
    auto count = [&](int64_t i, int64_t &as_wide, int64_t &as_narrow) {
        const Sequence n = sequence(a, (int32_t)i, false, bad);
        as_narrow = total_steps(a, n);
        as_wide = 0;
        if (can_be_wide(a, n)) as_wide = total_steps(a, sequence(a, (int32_t)i, true, ignore));
        sum[as_wide ? kEither : kNarrow] += as_narrow;
        sum[kWide] += as_wide;
    };
    const bool fits = __syncthreads_and(each <= kPlanKept);
#pragma unroll
    for (int x = 0; x < kPlanKept; ++x) {
        kept[x][0] = kept[x][1] = 0;
        if (fits && lo + x < hi) count(lo + x, kept[x][0], kept[x][1]);
    }
    if (!fits)
        for (int64_t i = lo; i < hi; ++i) {
            int64_t w, n;
            count(i, w, n);
        }
    const int lane = lane_id(), warp = threadIdx.x >> 5;
#pragma unroll
    for (int w = 0; w < kSums; ++w) {
        int64_t incl = sum[w];
#pragma unroll
        for (int d = 1; d < kWarp; d <<= 1) {
            const int64_t o = __shfl_up_sync(kFull, incl, d);
            if (lane >= d) incl += o;
        }
        if (lane == kWarp - 1) s_warp[w][warp] = incl;
        run[w] = incl - sum[w];
    }
    __syncthreads();
    // sums of the warps before this one, and of all: lane x has warp x's
#pragma unroll
    for (int w = 0; w < kSums; ++w) {
        all[w] = s_warp[w][lane];
        int64_t before = lane < warp ? all[w] : 0;
#pragma unroll
        for (int d = kWarp / 2; d > 0; d >>= 1) {
            before += __shfl_xor_sync(kFull, before, d);
            all[w] += __shfl_xor_sync(kFull, all[w], d);
        }
        run[w] += before;
    }
    const bool wide = a.n_wide > 0 && all[kEither] > (int64_t)kWideWorth * a.n_narrow;
    int64_t at_narrow = run[kNarrow] + (wide ? 0 : run[kEither]), at_wide = wide ? run[kWide] : 0;
    auto place = [&](int64_t i, int64_t as_wide, int64_t as_narrow) {
        a.start[0][i] = at_narrow;
        a.start[1][i] = at_wide;
        if (wide && as_wide) at_wide += as_wide;
        else at_narrow += as_narrow;
    };
#pragma unroll
    for (int x = 0; x < kPlanKept; ++x)
        if (fits && lo + x < hi) place(lo + x, kept[x][0], kept[x][1]);
    if (!fits)
        for (int64_t i = lo; i < hi; ++i) {
            const Sequence n = sequence(a, (int32_t)i, false, ignore);
            const bool can = can_be_wide(a, n);
            place(i, can ? total_steps(a, sequence(a, (int32_t)i, true, ignore)) : 0, total_steps(a, n));
        }
    if (threadIdx.x == 0) {
        const int64_t narrow = all[kNarrow] + (wide ? 0 : all[kEither]), wides = wide ? all[kWide] : 0;
        a.start[0][n] = narrow;
        a.start[1][n] = wides;
        a.start[0][n + 1] = max((int64_t)kNarrowMinSteps, (narrow + a.n_narrow - 1) / a.n_narrow);
        a.start[1][n + 1] = wide ? max((int64_t)1, (wides + a.n_wide - 1) / a.n_wide) : 1;
        a.start[1][n + 2] = wide ? 1 : 0;
    }
    const int64_t covered = __ldcg(a.group_offsets + a.N);
    for (int32_t r = threadIdx.x; r < a.R; r += kPlanThreads) {
        int32_t g = -1;
        if (r < covered) {
            int32_t l = 0, h = a.N - 1;                  // the last group that begins at or before r
            while (l < h) {
                const int32_t mid = (l + h + 1) >> 1;
                if ((in_shared ? s_off[mid] : __ldcg(a.group_offsets + mid)) <= r) l = mid;
                else h = mid - 1;
            }
            g = l;
        }
        a.group_of[r] = g;
    }
    if (bad) raise_status(a.status, HORA_ERR_INVALID_VALUE);
}

// Division of step numbers: 64-bit only where they need it.
__device__ __forceinline__ int32_t stream_of(int64_t u, int64_t per) {
    return ((u | per) >> 32) == 0 ? (int32_t)((uint32_t)u / (uint32_t)per) : (int32_t)(u / per);
}

// Joins the partials of the output rows: a warp to ROWS heads of a query and cache head, D / 32 neighbouring elements a lane.
// These rows' partials lie next to each other wherever they are (as long as they are of one item), so what is loaded for PARTS parts of
// an item is in flight together, and its place is worked out once.  With many rows eight of them and a part at a time; with few rows
// there may be dozens of parts to each, and one row with eight parts at a time is faster (one prompt of 103485 keys, 24
// rollouts, 37 parts a row: 147 us for the whole call with two rows and a part at a time, 125 so).
constexpr int kJoinRows = 8, kJoinParts = 8, kJoinWarps = 8;

template <typename T, int D, int ROWS, int PARTS>
__global__ void __launch_bounds__(256, 2)
attention_join_kernel(const AttnArgs a) {
    pdl_enter();
    constexpr int E = D / kWarp;
    const int lane = lane_id();
    const uint32_t chunks = (a.g + ROWS - 1) / ROWS, n_tasks = (uint32_t)a.R * a.T * a.Hkv * chunks;
    const uint32_t task = blockIdx.x * (blockDim.x / kWarp) + (threadIdx.x >> 5);
    if (task >= n_tasks) return;
    const uint32_t rth = task / chunks, g0 = (task - rth * chunks) * ROWS;
    const uint32_t rt = rth / a.Hkv, h = rth - rt * a.Hkv, r = rt / a.T, t = rt - r * a.T;
    const int32_t n = min(a.g - (int32_t)g0, ROWS);
    const int64_t rows = (int64_t)a.R * a.T * a.Hq, row = (int64_t)rt * a.Hq + h * a.g + g0;
    const int32_t grp = __ldcg(a.group_of + r);
    float m[ROWS], l[ROWS], o[ROWS][E];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        m[k] = -INFINITY;
        l[k] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[k][e] = 0.f;
    }
    if (grp >= 0 && (int32_t)t < query_count(a, r)) {
        bool bad = false;
        const bool wide = has_wide(a);
        const int64_t per_narrow = steps_per_stream<false>(a), per_wide = steps_per_stream<true>(a);
        const Sequence seq[2] = {sequence(a, grp, wide, bad), sequence(a, a.N + r, wide, bad)};
        const int64_t start[2][2] = {{__ldcg(a.start[0] + grp), __ldcg(a.start[1] + grp)}, {__ldcg(a.start[0] + a.N + r), __ldcg(a.start[1] + a.N + r)}};
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const Sequence &q = seq[part];
            if (q.steps == 0 || (int32_t)r < q.first || (int32_t)r >= q.first + q.rollouts) continue;
            const int64_t per = q.wide ? per_wide : per_narrow, first = q.wide ? start[part][1] : start[part][0];
            const int32_t stream_rows = q.wide ? kWideRows : a.narrow_rows;
            const float *cont_ml = q.wide ? a.cont_ml[1] : a.cont_ml[0], *cont_o = q.wide ? a.cont_o[1] : a.cont_o[0];
            uint32_t x = ((r - q.first) * a.T + t) * a.g + g0;
            for (int32_t j = 0; j < n;) {                // rows j .. j + count - 1 are of one item
                const uint32_t tile = x / (uint32_t)q.tile_rows, at = x - tile * q.tile_rows;
                const int32_t count = min(n - j, q.tile_rows - (int32_t)at);
                const int64_t u = first + ((int64_t)h * q.tiles + tile) * q.steps;
                const int32_t b0 = stream_of(u, per);
                const int64_t last = u - b0 * per + q.steps - 1;
                const int32_t more = last < per ? 0 : stream_of(last, per);
                // a wide item of one half has its keys dealt to two halves, each with a partial of its own
                const int halves = q.wide && min(q.tile_rows, q.rows - (int32_t)tile * q.tile_rows) <= kWideHalf ? 2 : 1;
                const int32_t parts = halves * (more + 1);
                for (int32_t p = 0; p < parts; p += PARTS) {
                    float2 ml[PARTS][ROWS];
                    float y[PARTS][ROWS][E];
#pragma unroll
                    for (int z = 0; z < PARTS; ++z) {
                        const int half = p + z > more ? 1 : 0;
                        const int32_t b = p + z - half * (more + 1);
                        const int64_t place = b == 0 ? (part + half * kSecondHalf) * rows + row + j : (int64_t)(b0 + b) * stream_rows + half * kWideHalf + at;
                        const bool have = p + z < parts && HORA_IN(place + count - 1, b == 0 ? 4 * rows : q.wide ? (int64_t)a.n_wide * kWideRows : (int64_t)a.n_narrow * a.narrow_rows);
                        const float2 *pml = reinterpret_cast<const float2 *>(b == 0 ? a.main_ml : cont_ml) + place - j;
                        const float *po = (b == 0 ? a.main_o : cont_o) + (place - j) * D + lane * E;
#pragma unroll
                        for (int k = 0; k < ROWS; ++k) {
                            ml[z][k] = make_float2(-INFINITY, 0.f);
#pragma unroll
                            for (int e = 0; e < E; ++e) y[z][k][e] = 0.f;
                            if (have && k >= j && k < j + count) {
                                ml[z][k] = __ldcg(pml + k);
                                if constexpr (E == 4) {
                                    const float4 v = __ldcg(reinterpret_cast<const float4 *>(po + k * D));
                                    y[z][k][0] = v.x; y[z][k][1] = v.y; y[z][k][2] = v.z; y[z][k][3] = v.w;
                                } else {
                                    const float2 v = __ldcg(reinterpret_cast<const float2 *>(po + k * D));
                                    y[z][k][0] = v.x; y[z][k][1] = v.y;
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int z = 0; z < PARTS; ++z)
#pragma unroll
                        for (int k = 0; k < ROWS; ++k) {
                            if (ml[z][k].x == -INFINITY) continue;          // no key seen there (and its output may not have been written)
                            const float top = fmaxf(m[k], ml[z][k].x), f = exp2_fast(m[k] - top), g = exp2_fast(ml[z][k].x - top);
                            m[k] = top;
                            l[k] = l[k] * f + ml[z][k].y * g;
#pragma unroll
                            for (int e = 0; e < E; ++e) o[k][e] = o[k][e] * f + y[z][k][e] * g;
                        }
                }
                j += count;
                x += count;
            }
        }
    }
    T *__restrict__ out = static_cast<T *>(a.out) + rt * a.out_row_stride + (int64_t)(h * a.g + g0) * D + lane * E;
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        if (k >= n) break;
        const float inv = m[k] == -INFINITY ? 0.f : 1.f / l[k];
        uint32_t w[E / 2];
#pragma unroll
        for (int e = 0; e < E; e += 2) w[e / 2] = pack2(o[k][e] * inv, o[k][e + 1] * inv, T());
        if constexpr (E == 4) *reinterpret_cast<uint2 *>(out + k * D) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(out + k * D) = w[0];
        if (a.lse != nullptr && lane == 0) a.lse[row + k] = m[k] == -INFINITY ? -INFINITY : 0.6931471805599453f * m[k] + logf(l[k]);
    }
}

static hora_status_t launch_plan(const AttnArgs &a, cudaStream_t stream) {
    const cudaError_t e = launch_pdl(attention_plan_kernel, 1, kPlanThreads, 0, stream, a);
    count_launches(1);
    return cuda_ok(e);
}

template <typename T, int D>
static cudaError_t launch_join_of(const AttnArgs &a, cudaStream_t stream) {
    const int64_t queries = (int64_t)a.R * a.T * a.Hkv;
    const bool many = queries >= (int64_t)a.n_sm * kJoinWarps;
    const int64_t tasks = queries * (many ? (a.g + kJoinRows - 1) / kJoinRows : a.g);
    return launch_pdl(many ? attention_join_kernel<T, D, kJoinRows, 1> : attention_join_kernel<T, D, 1, kJoinParts>, (int)((tasks + 7) / 8), 256, 0, stream, a);
}

static hora_status_t launch_join(const AttnArgs &a, int32_t q_dtype, int32_t D, cudaStream_t stream) {
    cudaError_t e;
    if (q_dtype == HORA_DTYPE_BF16) e = D == 64 ? launch_join_of<__nv_bfloat16, 64>(a, stream) : launch_join_of<__nv_bfloat16, 128>(a, stream);
    else e = D == 64 ? launch_join_of<__half, 64>(a, stream) : launch_join_of<__half, 128>(a, stream);
    count_launches(1);
    return cuda_ok(e);
}

// Places of the workspace, in order; returns the bytes used.
static size_t lay_out(AttnArgs &a, int32_t D, char *base) {
    size_t used = 0;
    auto take = [&](size_t bytes) {
        char *p = base + used;
        used += (bytes + 255) / 256 * 256;
        return p;
    };
    const size_t rows = (size_t)a.R * a.T * a.Hq;
    a.n_sm = sm_count();
    a.n_narrow = a.n_sm * kNarrowPerSm;
    a.narrow_rows = 8 * narrow_eights(a.T * a.g, D);
    a.n_wide = a.n_sm;
    for (int w = 0; w < 2; ++w) {
        const size_t cont = w ? (size_t)a.n_wide * kWideRows : (size_t)a.n_narrow * a.narrow_rows;
        a.start[w] = reinterpret_cast<int64_t *>(take(((size_t)a.N + a.R + 3) * 8));
        a.cont_o[w] = reinterpret_cast<float *>(take(cont * D * 4));
        a.cont_ml[w] = reinterpret_cast<float *>(take(cont * 2 * 4));
    }
    a.group_of = reinterpret_cast<int32_t *>(take((size_t)a.R * 4));
    a.main_o = reinterpret_cast<float *>(take(rows * 4 * D * 4));
    a.main_ml = reinterpret_cast<float *>(take(rows * 4 * 2 * 4));
    return used;
}

static bool sizes_ok(int64_t N, int64_t R, int32_t T, int32_t Hq, int32_t Hkv, int32_t D) {
    if (N < 0 || R < 0 || T < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || (D != 64 && D != 128)) return false;
    if (N > 0x3FFFFFFF || R > 0x3FFFFFFF || (R > 0 && N < 1)) return false;
    if ((int64_t)T * (Hq / Hkv) > 4096) return false;
    return R == 0 || (int64_t)T * Hq <= 0x7FFFFFFF / R;
}

}  // namespace hora

extern "C" size_t hora_group_attention_workspace_bytes(int64_t N, int64_t R, int32_t T, int32_t Hq, int32_t Hkv, int32_t D) {
    using namespace hora;
    if (!sizes_ok(N, R, T, Hq, Hkv, D)) return 0;
    AttnArgs a = {};
    a.N = (int32_t)N;
    a.R = (int32_t)R;
    a.T = T;
    a.Hq = Hq;
    a.g = Hq / Hkv;
    return lay_out(a, D, nullptr);
}

extern "C" hora_status_t hora_group_attention(const void *q, int32_t q_dtype, int64_t q_row_stride, const int64_t *group_offsets,
                                              int64_t N, int64_t R, int32_t T, const int32_t *q_len, int32_t Hq, int32_t Hkv,
                                              int32_t D, float sm_scale, const void *k_cache, const void *v_cache,
                                              const uint8_t *k_exp, const uint8_t *v_exp, int32_t cache_dtype, int64_t n_pages,
                                              int32_t page_size, const int32_t *prefix_pages, int32_t prefix_ld,
                                              const int32_t *prefix_len, const int32_t *suffix_pages, int32_t suffix_ld,
                                              const int32_t *suffix_len, void *out, int64_t out_row_stride, float *lse,
                                              int32_t *status_dev, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace hora;
    if (!sizes_ok(N, R, T, Hq, Hkv, D) || (q_dtype != HORA_DTYPE_BF16 && q_dtype != HORA_DTYPE_F16)) return HORA_ERR_INVALID_ARG;
    if (cache_dtype != q_dtype && cache_dtype != HORA_DTYPE_E4M3) return HORA_ERR_INVALID_ARG;
    if (!(sm_scale > 0.f) || sm_scale > 1e30f) return HORA_ERR_INVALID_ARG;
    if (prefix_ld < 0 || suffix_ld < 0 || (int64_t)prefix_ld * page_size > 0x7FFFFF00 || (int64_t)suffix_ld * page_size > 0x7FFFFF00)
        return HORA_ERR_INVALID_ARG;
    if (R == 0) return HORA_OK;
    if (!cache_ok(k_cache, v_cache, k_exp, v_exp, cache_dtype, n_pages, page_size, Hkv, D)) return HORA_ERR_INVALID_ARG;
    if (q == nullptr || out == nullptr || group_offsets == nullptr || prefix_len == nullptr || suffix_len == nullptr) return HORA_ERR_INVALID_ARG;
    if ((prefix_pages == nullptr && prefix_ld > 0) || (suffix_pages == nullptr && suffix_ld > 0)) return HORA_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15u) return HORA_ERR_INVALID_ARG;
    const int64_t width = (int64_t)Hq * D;
    if (q_row_stride < width || q_row_stride % 8 || out_row_stride < width || out_row_stride % 8) return HORA_ERR_INVALID_ARG;
    AttnArgs a = {};
    a.N = (int32_t)N;
    a.R = (int32_t)R;
    a.T = T;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.g = Hq / Hkv;
    if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HORA_ERR_WORKSPACE;
    if (lay_out(a, D, static_cast<char *>(workspace)) > workspace_bytes) return HORA_ERR_WORKSPACE;
    a.q = q;
    a.group_offsets = group_offsets;
    a.q_len = q_len;
    a.prefix_pages = prefix_pages;
    a.prefix_len = prefix_len;
    a.suffix_pages = suffix_pages;
    a.suffix_len = suffix_len;
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.k_exp = k_exp;
    a.v_exp = v_exp;
    a.out = out;
    a.lse = lse;
    a.status = status_dev;
    a.q_row_stride = q_row_stride;
    a.out_row_stride = out_row_stride;
    a.n_pages = n_pages;
    a.page_shift = page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7;
    a.prefix_ld = prefix_ld;
    a.suffix_ld = suffix_ld;
    a.scale_log2 = sm_scale * 1.4426950408889634f;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cache_dtype == HORA_DTYPE_E4M3) a.n_wide = 0;
    a.narrow_keys = narrow_keys(cache_dtype == HORA_DTYPE_E4M3, D);
    hora_status_t rc = launch_plan(a, s);
    if (rc == HORA_OK) rc = launch_attention_main(a, q_dtype, cache_dtype, D, s);
    if (rc == HORA_OK) rc = launch_join(a, q_dtype, D, s);
    return rc;
}
