// hora_kv_write / hora_kv_read: rows of keys and values into and out of the paged cache, quantised on the way.
//
// A row (one token, one head, D elements) belongs to D/8 neighbouring lanes, eight elements each: one 16-byte access a
// lane on the 16-bit side, the row's largest magnitude by log2(D/8) shuffles, one 8-byte access on the e4m3 side.  The scale of
// a quantised row is a power of two, so x / 2^e is exact and the code is the one rounding of the definition.  Nothing is
// reused: the calls are bound by HBM.  Slots are read by ordinary loads, which L1 serves to the other heads of a token (through L2 the same took a
// tenth longer).  Every lane group has kRowsInFlight rows' loads in flight before it converts the first.
#include <type_traits>

#include "hora_rows16.cuh"

namespace hora {

constexpr int kKvThreads = 128;                          // 131072 tokens (below): 291 us with 128, 316 with 256
constexpr int kRowsInFlight = 4;                         // 131072 tokens, 8 heads of 128, bf16 -> e4m3 -> bf16: 291 us (5.5 TB/s; 310 on another GPU); 306 with 2, 296 with 8

struct KvShape {
    int64_t n_tokens, row_stride, n_slots;
    int32_t H, page_shift, tokens_per_cta;
};

// Where the row of slot `slot`, head h, begins in a pool (in rows).
__device__ __forceinline__ int64_t pool_row(int64_t slot, int32_t h, const KvShape &s) {
    const int64_t page = slot >> s.page_shift, at = slot & ((1 << s.page_shift) - 1);
    return ((page * s.H + h) << s.page_shift) + at;
}

// The rows of a CTA's tokens, dealt to its lane groups in order (token-major), kRowsInFlight at a time.
template <int GROUPS>
struct RowWalk {
    int32_t t, h, dt, dh, H;
    __device__ RowWalk(int group, int32_t H_) : H(H_) {
        t = group / H;
        h = group - t * H;
        dt = GROUPS / H;
        dh = GROUPS - dt * H;
    }
    __device__ void next() {
        t += dt;
        h += dh;
        if (h >= H) { h -= H; ++t; }
    }
};

template <typename In, typename Cache, int D>
__global__ void __launch_bounds__(kKvThreads)
kv_write_kernel(const In *k, const In *v, const int64_t *slots, KvShape s,
                Cache *__restrict__ k_cache, Cache *__restrict__ v_cache, uint8_t *__restrict__ k_exp,
                uint8_t *__restrict__ v_exp, int32_t *status) {
    pdl_enter();
    constexpr int kLanes = D / 8, kGroups = kKvThreads / kLanes;
    const int sub = threadIdx.x % kLanes;
    const In *in = blockIdx.y == 0 ? k : v;
    Cache *__restrict__ cache = blockIdx.y == 0 ? k_cache : v_cache;
    uint8_t *__restrict__ exps = blockIdx.y == 0 ? k_exp : v_exp;
    const int64_t t0 = (int64_t)blockIdx.x * s.tokens_per_cta;
    const int64_t left = s.n_tokens - t0;
    const int32_t n_tok = left < s.tokens_per_cta ? (int32_t)left : s.tokens_per_cta;
    RowWalk<kGroups> w(threadIdx.x / kLanes, s.H);
    // the lane groups of a warp leave together: the shuffles below need all of them
    for (int base = 0; base < n_tok * s.H; base += kRowsInFlight * kGroups) {
        Raw8<In> raw[kRowsInFlight];
        int64_t slot[kRowsInFlight];
        int32_t head[kRowsInFlight];
#pragma unroll
        for (int u = 0; u < kRowsInFlight; ++u) {
            slot[u] = -1;
            head[u] = w.h;
            zero8(raw[u]);
            if (w.t < n_tok) {
                slot[u] = slots[t0 + w.t];
                load8(raw[u], in + (t0 + w.t) * s.row_stride + w.h * D + sub * 8);
            }
            w.next();
        }
#pragma unroll
        for (int u = 0; u < kRowsInFlight; ++u) {
            const bool beyond = slot[u] >= s.n_slots;
            if (beyond && sub == 0) raise_status(status, HORA_ERR_INVALID_VALUE);
            const bool keep = slot[u] >= 0 && !beyond;
            const int64_t row = keep ? pool_row(slot[u], head[u], s) : 0;
            float x[8];
            widen8(raw[u], x);
            if constexpr (sizeof(Cache) == 1) {
                float a = largest8(raw[u]);
                if (!(a <= 3.402823466e38f)) {                             // not finite: the largest of those that are
                    a = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) a = fabsf(x[i]) <= 3.402823466e38f ? fmaxf(a, fabsf(x[i])) : a;
                }
#pragma unroll
                for (int d = kLanes / 2; d > 0; d >>= 1) a = fmaxf(a, __shfl_xor_sync(kFull, a, d));
                // a = m 2^x, 1 <= m < 2;  448 = 1.75 * 2^8: e = x - 8, one more where m > 1.75
                const uint32_t bits = __float_as_uint(a);
                int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
                e = bits == 0u ? 0 : (e < -126 ? -126 : e);
                const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] *= inv;
                if (keep && sub == 0) exps[row] = (uint8_t)(e + 127);
            }
            Raw8<Cache> o;
            narrow8(x, o);
            if (keep) store8(o, cache + row * D + sub * 8);
        }
    }
}

template <typename Out, typename Cache, int D>
__global__ void __launch_bounds__(kKvThreads)
kv_read_kernel(const Cache *k_cache, const Cache *v_cache, const uint8_t *k_exp,
               const uint8_t *v_exp, const int64_t *slots, KvShape s, Out *__restrict__ k,
               Out *__restrict__ v, int32_t *status) {
    pdl_enter();
    constexpr int kLanes = D / 8, kGroups = kKvThreads / kLanes;
    const int sub = threadIdx.x % kLanes;
    const Cache *cache = blockIdx.y == 0 ? k_cache : v_cache;
    const uint8_t *exps = blockIdx.y == 0 ? k_exp : v_exp;
    Out *__restrict__ out = blockIdx.y == 0 ? k : v;
    const int64_t t0 = (int64_t)blockIdx.x * s.tokens_per_cta;
    const int64_t left = s.n_tokens - t0;
    const int32_t n_tok = left < s.tokens_per_cta ? (int32_t)left : s.tokens_per_cta;
    RowWalk<kGroups> w(threadIdx.x / kLanes, s.H);
    while (w.t < n_tok) {
        Raw8<Cache> raw[kRowsInFlight];
        int64_t to[kRowsInFlight];
        int32_t e[kRowsInFlight];
#pragma unroll
        for (int u = 0; u < kRowsInFlight; ++u) {
            to[u] = -1;
            e[u] = 127;
            zero8(raw[u]);
            if (w.t < n_tok) {
                to[u] = (t0 + w.t) * s.row_stride + w.h * D + sub * 8;
                const int64_t slot = slots[t0 + w.t];
                if (slot >= s.n_slots) {
                    if (sub == 0) raise_status(status, HORA_ERR_INVALID_VALUE);
                } else if (slot >= 0) {
                    const int64_t row = pool_row(slot, w.h, s);
                    load8(raw[u], cache + row * D + sub * 8);
                    if constexpr (sizeof(Cache) == 1) e[u] = __ldcg(exps + row);
                }
            }
            w.next();
        }
#pragma unroll
        for (int u = 0; u < kRowsInFlight; ++u) {
            if (to[u] < 0) continue;
            float x[8];
            widen8(raw[u], x);
            if constexpr (sizeof(Cache) == 1) {
                // 2^(e-127): the byte is the exponent field of the scale (0 stands for 2^-127)
                const float scale = e[u] ? __uint_as_float((uint32_t)e[u] << 23) : __uint_as_float(0x400000u);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] *= scale;
            }
            Raw8<Out> o;
            narrow8(x, o);
            store8(o, out + to[u]);
        }
    }
}

static KvShape kv_shape(int64_t n_tokens, int32_t H, int64_t row_stride, int64_t n_pages, int32_t page_size, int D, int *grid) {
    KvShape s;
    s.n_tokens = n_tokens;
    s.row_stride = row_stride;
    s.n_slots = n_pages * page_size;
    s.H = H;
    s.page_shift = page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7;
    // a CTA takes two rounds of its lane groups' rows, fewer when that would leave multiprocessors without work
    const int64_t round = kRowsInFlight * (kKvThreads / (D / 8));
    int64_t tok = (2 * round + H - 1) / H;
    const int64_t spread = (n_tokens * 2 + sm_count() - 1) / sm_count();
    if (tok > spread) tok = spread;
    if (tok < 1) tok = 1;
    while ((n_tokens + tok - 1) / tok > 0x7FFFFFFF) tok *= 2;
    s.tokens_per_cta = (int32_t)tok;
    *grid = (int)((n_tokens + tok - 1) / tok);
    return s;
}

template <typename... KArgs, typename... Args>
static hora_status_t launch_kv(void (*kernel)(KArgs...), int grid, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid, 2);
    cfg.blockDim = dim3(kKvThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
    count_launches(1);
    return cuda_ok(e);
}

static bool rows_ok(const void *k, const void *v, int32_t dtype, int64_t row_stride, int32_t H, int32_t D) {
    if (dtype != HORA_DTYPE_F32 && dtype != HORA_DTYPE_BF16 && dtype != HORA_DTYPE_F16) return false;
    if (k == nullptr || v == nullptr || ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u)) return false;
    return row_stride >= (int64_t)H * D && row_stride < (1LL << 40) && (row_stride * dtype_bytes(dtype)) % 16 == 0;
}

// Calls f with null pointers of the row type and the cache type, and the head size as a constant.
template <typename F>
static hora_status_t kv_dispatch(int32_t row_dtype, int32_t cache_dtype, int32_t D, F &&f) {
    auto by_d = [&](auto row, auto cache) {
        return D == 64 ? f(row, cache, std::integral_constant<int, 64>()) : f(row, cache, std::integral_constant<int, 128>());
    };
    auto by_cache = [&](auto row) {
        switch (cache_dtype) {
            case HORA_DTYPE_BF16: return by_d(row, (__nv_bfloat16 *)nullptr);
            case HORA_DTYPE_F16: return by_d(row, (__half *)nullptr);
            default: return by_d(row, (E4M3 *)nullptr);
        }
    };
    switch (row_dtype) {
        case HORA_DTYPE_F32: return by_cache((float *)nullptr);
        case HORA_DTYPE_BF16: return by_cache((__nv_bfloat16 *)nullptr);
        default: return by_cache((__half *)nullptr);
    }
}

}  // namespace hora

extern "C" hora_status_t hora_kv_write(const void *k, const void *v, int32_t in_dtype, int64_t in_row_stride, const int64_t *slots,
                                       int64_t n_tokens, int32_t H, int32_t D, void *k_cache, void *v_cache, uint8_t *k_exp,
                                       uint8_t *v_exp, int32_t cache_dtype, int64_t n_pages, int32_t page_size,
                                       int32_t *status_dev, void *stream) {
    using namespace hora;
    if (n_tokens < 0 || H < 1 || H > 4096) return HORA_ERR_INVALID_ARG;
    if (n_tokens == 0) return HORA_OK;
    if (slots == nullptr || !rows_ok(k, v, in_dtype, in_row_stride, H, D)) return HORA_ERR_INVALID_ARG;
    if (!cache_ok(k_cache, v_cache, k_exp, v_exp, cache_dtype, n_pages, page_size, H, D)) return HORA_ERR_INVALID_ARG;
    int grid;
    const KvShape s = kv_shape(n_tokens, H, in_row_stride, n_pages, page_size, D, &grid);
    return kv_dispatch(in_dtype, cache_dtype, D, [&](auto *row, auto *cache, auto d) {
        using In = std::remove_pointer_t<decltype(row)>;
        using Cache = std::remove_pointer_t<decltype(cache)>;
        return launch_kv(kv_write_kernel<In, Cache, decltype(d)::value>, grid, static_cast<cudaStream_t>(stream), static_cast<const In *>(k),
                         static_cast<const In *>(v), slots, s, static_cast<Cache *>(k_cache), static_cast<Cache *>(v_cache), k_exp,
                         v_exp, status_dev);
    });
}

extern "C" hora_status_t hora_kv_read(const void *k_cache, const void *v_cache, const uint8_t *k_exp, const uint8_t *v_exp,
                                      int32_t cache_dtype, int64_t n_pages, int32_t page_size, const int64_t *slots, int64_t n_tokens,
                                      int32_t H, int32_t D, void *k, void *v, int32_t out_dtype, int64_t out_row_stride,
                                      int32_t *status_dev, void *stream) {
    using namespace hora;
    if (n_tokens < 0 || H < 1 || H > 4096) return HORA_ERR_INVALID_ARG;
    if (n_tokens == 0) return HORA_OK;
    if (slots == nullptr || !rows_ok(k, v, out_dtype, out_row_stride, H, D)) return HORA_ERR_INVALID_ARG;
    if (!cache_ok(k_cache, v_cache, k_exp, v_exp, cache_dtype, n_pages, page_size, H, D)) return HORA_ERR_INVALID_ARG;
    int grid;
    const KvShape s = kv_shape(n_tokens, H, out_row_stride, n_pages, page_size, D, &grid);
    return kv_dispatch(out_dtype, cache_dtype, D, [&](auto *row, auto *cache, auto d) {
        using Out = std::remove_pointer_t<decltype(row)>;
        using Cache = std::remove_pointer_t<decltype(cache)>;
        return launch_kv(kv_read_kernel<Out, Cache, decltype(d)::value>, grid, static_cast<cudaStream_t>(stream),
                         static_cast<const Cache *>(k_cache), static_cast<const Cache *>(v_cache), k_exp, v_exp, slots, s,
                         static_cast<Out *>(k), static_cast<Out *>(v), status_dev);
    });
}
