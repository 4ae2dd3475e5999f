// hora_group_attention: plan, joining of the partial results, and the C entry.
#include "hora_group_attention.cuh"

namespace hora {

constexpr int kPlanThreads = 1024;
constexpr int kWideFrom = 33;

// start[line][i] = steps before sequence i on its line, group_of[r].  One CTA: every thread takes a run of sequences.
__global__ void __launch_bounds__(kPlanThreads)
attention_plan_kernel(const AttnArgs a) {
    pdl_enter();
    __shared__ int64_t s_warp[2][kPlanThreads / kWarp];
    const int64_t n = (int64_t)a.N + a.R;
    const int64_t each = (n + kPlanThreads - 1) / kPlanThreads;
    const int64_t lo = min(n, each * threadIdx.x), hi = min(n, lo + each);
    bool bad = false;
    int64_t sum[2] = {0, 0}, run[2];
    for (int64_t i = lo; i < hi; ++i) {
        const Sequence s = sequence(a, (int32_t)i, bad);
        (s.wide ? sum[1] : sum[0]) += total_steps(a, s);
    }
    const int lane = lane_id(), warp = threadIdx.x >> 5;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
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
#pragma unroll
    for (int w = 0; w < 2; ++w)
        for (int x = 0; x < warp; ++x) run[w] += s_warp[w][x];
    for (int64_t i = lo; i < hi; ++i) {
        a.start[0][i] = run[0];
        a.start[1][i] = run[1];
        bool again = false;
        const Sequence s = sequence(a, (int32_t)i, again);
        (s.wide ? run[1] : run[0]) += total_steps(a, s);
    }
    if (threadIdx.x == kPlanThreads - 1) {
        a.start[0][n] = run[0];
        a.start[1][n] = run[1];
    }
    const int64_t covered = __ldg(a.group_offsets + a.N);
    for (int32_t r = threadIdx.x; r < a.R; r += kPlanThreads) {
        int32_t g = -1;
        if (r < covered) {
            int32_t l = 0, h = a.N - 1;                  // the last group that begins at or before r
            while (l < h) {
                const int32_t mid = (l + h + 1) >> 1;
                if (__ldg(a.group_offsets + mid) <= r) l = mid;
                else h = mid - 1;
            }
            g = l;
        }
        a.group_of[r] = g;
    }
    if (bad) raise_status(a.status, HORA_ERR_INVALID_VALUE);
}

// Joins the partials of one output row; a warp to a row, D / 32 neighbouring elements a lane.
template <int E>
struct Joined {
    float m = -INFINITY, l = 0.f, o[E] = {};

    __device__ __forceinline__ void add(float m2, float l2, const float *__restrict__ p, int lane) {
        if (m2 == -INFINITY) return;                     // no key of that part is seen
        const float top = fmaxf(m, m2), f = exp2f(m - top), f2 = exp2f(m2 - top);
        l = l * f + l2 * f2;
        float x[E];
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float2 y = __ldcs(reinterpret_cast<const float2 *>(p + lane * E + e));
            x[e] = y.x;
            x[e + 1] = y.y;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + x[e] * f2;
        m = top;
    }
};

template <typename T, int D>
__global__ void __launch_bounds__(256)
attention_join_kernel(const AttnArgs a) {
    pdl_enter();
    constexpr int E = D / kWarp;
    const int lane = lane_id();
    const int64_t rows = (int64_t)a.R * a.T * a.Hq;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / kWarp) + (threadIdx.x >> 5);
    if (row >= rows) return;
    const int32_t head = (int32_t)(row % a.Hq);
    const int64_t rt = row / a.Hq;
    const int32_t r = (int32_t)(rt / a.T), t = (int32_t)(rt % a.T), h = head / a.g;
    Joined<E> j;
    const int32_t grp = a.group_of[r];
    if (grp >= 0 && t < query_count(a, r)) {
        bool bad = false;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const int32_t i = part == kPromptPart ? grp : a.N + r;
            const Sequence s = sequence(a, i, bad);
            if (s.steps == 0 || r < s.first || r >= s.first + s.rollouts) continue;
            const int32_t x = ((r - s.first) * a.T + t) * a.g + head % a.g;
            const int32_t tile = x / s.tile_rows, at = x % s.tile_rows;
            const int64_t u0 = __ldg(a.start[s.wide] + i) + ((int64_t)h * s.tiles + tile) * s.steps;
            const int64_t per = s.wide ? steps_per_stream<true>(a) : steps_per_stream<false>(a);
            // a wide item of one half has its keys dealt to two halves, each with a partial of its own
            const int halves = s.wide && min(s.tile_rows, s.rows - tile * s.tile_rows) <= kWideHalf ? 2 : 1;
            const int32_t b0 = (int32_t)(u0 / per), b1 = (int32_t)((u0 + s.steps - 1) / per);
            for (int half = 0; half < halves; ++half) {
                const int64_t place = (part + half * kSecondHalf) * rows + row;
                const float2 ml = *reinterpret_cast<const float2 *>(a.main_ml + place * 2);
                j.add(ml.x, ml.y, a.main_o + place * D, lane);
                for (int32_t b = b0 + 1; b <= b1; ++b) {
                    const int64_t c = (int64_t)b * (s.wide ? kWideRows : kNarrowRows) + half * kWideHalf + at;
                    const float2 ml2 = *reinterpret_cast<const float2 *>(a.cont_ml[s.wide] + c * 2);
                    j.add(ml2.x, ml2.y, a.cont_o[s.wide] + c * D, lane);
                }
            }
        }
    }
    const float inv = j.l > 0.f ? 1.f / j.l : (j.m == -INFINITY ? 0.f : 1.f / j.l);
    T *__restrict__ out = static_cast<T *>(a.out) + rt * a.out_row_stride + (int64_t)head * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2) *reinterpret_cast<uint32_t *>(out + e) = pack2(j.o[e] * inv, j.o[e + 1] * inv, T());
    if (a.lse != nullptr && lane == 0) a.lse[row] = j.m == -INFINITY ? -INFINITY : 0.6931471805599453f * j.m + logf(j.l);
}

static hora_status_t launch_plan(const AttnArgs &a, cudaStream_t stream) {
    const cudaError_t e = launch_pdl(attention_plan_kernel, 1, kPlanThreads, 0, stream, a);
    count_launches(1);
    return cuda_ok(e);
}

static hora_status_t launch_join(const AttnArgs &a, int32_t q_dtype, int32_t D, cudaStream_t stream) {
    const int64_t rows = (int64_t)a.R * a.T * a.Hq;
    const int grid = (int)((rows + 7) / 8);
    cudaError_t e;
    if (q_dtype == HORA_DTYPE_BF16)
        e = D == 64 ? launch_pdl(attention_join_kernel<__nv_bfloat16, 64>, grid, 256, 0, stream, a)
                    : launch_pdl(attention_join_kernel<__nv_bfloat16, 128>, grid, 256, 0, stream, a);
    else
        e = D == 64 ? launch_pdl(attention_join_kernel<__half, 64>, grid, 256, 0, stream, a)
                    : launch_pdl(attention_join_kernel<__half, 128>, grid, 256, 0, stream, a);
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
    a.n_narrow = sm_count() * kNarrowPerSm;
    a.n_wide = sm_count();
    for (int w = 0; w < 2; ++w) {
        const size_t cont = w ? (size_t)a.n_wide * kWideRows : (size_t)a.n_narrow * kNarrowRows;
        a.start[w] = reinterpret_cast<int64_t *>(take(((size_t)a.N + a.R + 1) * 8));
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
    a.wide_from = kWideFrom;
    hora_status_t rc = launch_plan(a, s);
    if (rc == HORA_OK) rc = launch_attention_narrow(a, q_dtype, cache_dtype, D, s);
    if (rc == HORA_OK && a.n_wide > 0) rc = launch_attention_wide(a, q_dtype, D, s);
    if (rc == HORA_OK) rc = launch_join(a, q_dtype, D, s);
    return rc;
}
