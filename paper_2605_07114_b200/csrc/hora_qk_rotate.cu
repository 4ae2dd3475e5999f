// hora_qk_rotate, hora_qk_rotate_backward: norms of queries and keys for each head with the position rotation in the same pass.
//
//   r = 1 / sqrt(mean x^2 + eps), z = x r w, y = R z      R turns the pairs (a, b) of z: (a cos - b sin, a sin + b cos)
//   g = R^T dy, dx = r (w g - x r mean(x r w g)), dw = sum over rows of x r g
//
// A row (one token, one head) lies in D / 8 neighbouring lanes, eight values each, so the mean is three or four shuffles and the
// other value of a pair (i, i + rot/2) one more.  Such a group of lanes takes one token and several of its heads, one after the other: the
// angles are worked out once for all of them, in 64 bits up to the fraction of a turn (a position of 10^5 times a frequency of 1
// has lost 2^-8 of a radian in 32 bits), the weights are held in registers, and four heads' loads are in flight.
//   What bounds it: HBM and issue slots, about equally.  Nothing is read twice and nothing but the results is written: 131072 tokens of 20 heads of 128 in
// bf16 254 us, 5.3 TB/s (0.81 of the copy rate) where inputs stay from pass to pass, 272 to 283 where they change; 50021 tokens of 32 heads and back 396
// and 403 to 420 us, 5.2 TB/s; seven of ten cycles issuing.  The forward kernels of 16-bit types are held to 80 registers, so that three CTAs fit an SM,
// for which they spill 12 (neighbouring pairs) to 68 bytes a thread; of the backward ones, held to 128, those of fp32 do, 8 to 56.
#define HORA_FILE_ID 8
#include "hora_rows16.cuh"

namespace hora {

constexpr int kRotateThreads = 256;
constexpr int kRotateHeads = 4;                          // heads whose loads are in flight together
constexpr int kRotateUnits = 9472;                       // groups of lanes that fill the device: 148 * 8 warps of two, four times over
constexpr int kRotatePerSm = 4;                          // CTAs of the backward pass an SM; each has a place for its part of the weights' gradients

struct RotateArgs {
    const void *x[2], *dy[2];                            // queries, keys
    void *y[2];                                          // what is written: y, or dx
    const float *w[2];
    int64_t x_stride[2], dy_stride[2], y_stride[2];
    const int32_t *positions;
    const double *inv_freq;
    int64_t units;
    int32_t Hq, H, chunks, heads;                        // heads of a chunk
    int32_t rot;
    float eps;
    float *parts;                                        // [CTAs][2][D]
};

template <int LANES>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
    return v;
}

// Cosines and sines of a lane's eight values; the sine's sign is that of its place in the pair, times `way` (-1: backwards).
// `other`: how far away the lane with the other values of the pairs is (0 with neighbouring pairs, whose four angles come twice).
template <int D, bool PAIRS>
struct Turn {
    float c[8], s[8];
    int other;
    bool turned;

    __device__ __forceinline__ Turn(const RotateArgs &a, int64_t token, bool have, int lane, float way) {
        const int e0 = lane * 8, half = a.rot / 2;
        turned = have && e0 < a.rot;
        const bool first = PAIRS || e0 < half;
        other = PAIRS || e0 >= a.rot ? 0 : first ? half / 8 : -(half / 8);
        const double at = turned ? (double)__ldcg(a.positions + token) : 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (PAIRS && (i & 1)) continue;
            const int f = PAIRS ? (e0 + i) / 2 : first ? e0 + i : e0 - half + i;
            const double turns = turned ? at * (__ldca(a.inv_freq + f) * 0.15915494309189535) : 0.0;
            float sn, cs;
            sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
            sn *= way;
            if constexpr (PAIRS) {
                c[i] = c[i + 1] = cs;
                s[i] = -sn;
                s[i + 1] = sn;
            } else {
                c[i] = cs;
                s[i] = first ? -sn : sn;
            }
        }
    }
};

// The eight values of the lane `other` away, as they lie in memory.  All lanes of the warp.
__device__ __forceinline__ uint4 shuffled(const uint4 &v, int from) {
    return make_uint4(__shfl_sync(kFull, v.x, from), __shfl_sync(kFull, v.y, from), __shfl_sync(kFull, v.z, from), __shfl_sync(kFull, v.w, from));
}
__device__ __forceinline__ float4 shuffled(const float4 &v, int from) {
    return make_float4(__shfl_sync(kFull, v.x, from), __shfl_sync(kFull, v.y, from), __shfl_sync(kFull, v.z, from), __shfl_sync(kFull, v.w, from));
}
template <typename T>
__device__ __forceinline__ Raw8<T> shuffled(const Raw8<T> &v, int from) {
    Raw8<T> r;
    r.a = shuffled(v.a, from);
    if constexpr (sizeof(Raw8<T>) == 32) r.b = shuffled(v.b, from);
    return r;
}
template <typename T, bool PAIRS>
__device__ __forceinline__ void others8(const Raw8<T> &v, const float (&x)[8], int from, float (&p)[8]) {
    if constexpr (PAIRS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = x[i ^ 1];
    } else {
        widen8(shuffled(v, from), p);
    }
}

// One group's heads of one side, from..to - 1 of it: x (and dy) at a token's first head, the result to y.  The next heads' loads are on their
// way while these are worked on; `first` has been called before the angles were worked out.  The weights enter the angles' cosines and sines once for
// all heads; what a lane takes from the other lane of its pairs it takes as it lies in memory (the kernels issue in 0.7 of the cycles: their
// instructions count).
template <typename T, int D, bool PAIRS, bool BACKWARD>
struct Side {
    static constexpr int kLanes = D / 8, kAhead = BACKWARD ? kRotateHeads / 2 : kRotateHeads;
    const T *x, *dy;
    T *y;
    int32_t from, to;
    bool norm;
    Raw8<T> next_x[kAhead], next_dy[kAhead];

    __device__ __forceinline__ void load(int32_t h) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (h + i < to && (!BACKWARD || norm)) load8(next_x[i], x + (h + i) * D);
            else zero8(next_x[i]);
            if constexpr (BACKWARD) {
                if (h + i < to) load8(next_dy[i], dy + (h + i) * D);
                else zero8(next_dy[i]);
            }
        }
    }

    // `most`: heads of the warp's group with the most
    __device__ __forceinline__ void run(const Turn<D, PAIRS> &turn, const float (&w)[8], float (&dw)[8], float eps, int lane_in_warp, int32_t most) {
        const int source = lane_in_warp + turn.other;
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // forwards the weights of both values of a pair enter: r (x w c + x' w' s)
            const float other_w = BACKWARD ? 1.f : PAIRS ? w[i ^ 1] : __shfl_sync(kFull, w[i], source);
            c[i] = BACKWARD ? turn.c[i] : turn.c[i] * w[i];
            s[i] = BACKWARD ? turn.s[i] : turn.s[i] * other_w;
        }
#pragma unroll 1
        for (int32_t b = 0; b < most; b += kAhead) {
            Raw8<T> now_x[kAhead], now_dy[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                now_x[i] = next_x[i];
                if (BACKWARD) now_dy[i] = next_dy[i];
            }
            const int32_t h = from + b;
            load(h + kAhead);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (b + i >= most) break;
                float z[8], p[8];
                float r = 1.f;
                widen8(now_x[i], z);
                if (norm) {                              // alike for the whole warp
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += z[e] * z[e];
                    r = rsqrtf(group_sum<kLanes>(sum) * (1.f / D) + eps);
                    // lanes with no head left hold zeros, whose r is infinite where eps is 0: infinity times zero would be in dw
                    if (BACKWARD && h + i >= to) r = 0.f;
                }
                if constexpr (!BACKWARD) {
                    others8<T, PAIRS>(now_x[i], z, source, p);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        z[e] *= c[e];
                        if (turn.turned) z[e] += p[e] * s[e];
                        z[e] *= r;
                    }
                } else {
                    float g[8];
                    widen8(now_dy[i], g);
                    others8<T, PAIRS>(now_dy[i], g, source, p);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        g[e] *= c[e];
                        if (turn.turned) g[e] += p[e] * s[e];
                    }
                    if (norm) {
                        float dot = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            dw[e] += r * z[e] * g[e];
                            g[e] *= w[e];
                            dot += z[e] * g[e];
                        }
                        dot = group_sum<kLanes>(dot) * (1.f / D) * r * r;
#pragma unroll
                        for (int e = 0; e < 8; ++e) g[e] = r * (g[e] - z[e] * dot);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = g[e];
                }
                if (h + i < to) {
                    Raw8<T> out;
                    narrow8(z, out);
                    store8(out, y + (h + i) * D);
                }
            }
        }
    }
};

// One group's part: a token and `heads` of its heads.
template <typename T, int D, bool PAIRS, bool BACKWARD>
__device__ __forceinline__ void rotate_unit(const RotateArgs &a, int64_t unit, bool have, const float (&w)[2][8], float (&dw)[2][8]) {
    constexpr int kLanes = D / 8;
    const int lane_in_warp = lane_id(), lane = lane_in_warp % kLanes;
    const int64_t token = have ? (a.chunks == 1 ? unit : unit / a.chunks) : 0;
    const int32_t h0 = have && a.chunks > 1 ? (int32_t)(unit - token * a.chunks) * a.heads : 0, h1 = have ? min(a.H, h0 + a.heads) : h0;
    auto side = [&](int k) {
        Side<T, D, PAIRS, BACKWARD> s;
        s.x = static_cast<const T *>(k ? a.x[1] : a.x[0]) + token * (k ? a.x_stride[1] : a.x_stride[0]) + lane * 8;
        s.dy = static_cast<const T *>(k ? a.dy[1] : a.dy[0]) + token * (k ? a.dy_stride[1] : a.dy_stride[0]) + lane * 8;
        s.y = static_cast<T *>(k ? a.y[1] : a.y[0]) + token * (k ? a.y_stride[1] : a.y_stride[0]) + lane * 8;
        s.from = k ? max(h0 - a.Hq, 0) : h0;
        s.to = k ? max(h1 - a.Hq, s.from) : max(min(h1, a.Hq), h0);
        s.norm = (k ? a.w[1] : a.w[0]) != nullptr;
        return s;
    };
    Side<T, D, PAIRS, BACKWARD> q = side(0);
    q.load(q.from);
    const Turn<D, PAIRS> turn(a, token, have, lane, BACKWARD ? -1.f : 1.f);
    int32_t most = __reduce_max_sync(kFull, q.to - q.from);
    if (most > 0) q.run(turn, w[0], dw[0], a.eps, lane_in_warp, most);
    Side<T, D, PAIRS, BACKWARD> k = side(1);
    most = __reduce_max_sync(kFull, k.to - k.from);
    if (most > 0) {
        k.load(k.from);
        k.run(turn, w[1], dw[1], a.eps, lane_in_warp, most);
    }
}

template <int D>
__device__ __forceinline__ void load_weights(const RotateArgs &a, float (&w)[2][8]) {
    const int lane = lane_id() % (D / 8);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) w[s][e] = a.w[s] ? __ldca(a.w[s] + lane * 8 + e) : 1.f;
}

template <typename T, int D, bool PAIRS>
__global__ void __launch_bounds__(kRotateThreads, sizeof(T) == 2 ? 3 : 2)
qk_rotate_kernel(const RotateArgs a) {
    pdl_enter();
    constexpr int kGroups = kRotateThreads / (D / 8);
    float w[2][8], dw[2][8];
    load_weights<D>(a, w);
    const int64_t unit = (int64_t)blockIdx.x * kGroups + threadIdx.x / (D / 8);
    rotate_unit<T, D, PAIRS, false>(a, unit, unit < a.units, w, dw);
}

template <typename T, int D, bool PAIRS>
__global__ void __launch_bounds__(kRotateThreads, 2)
qk_rotate_backward_kernel(const RotateArgs a) {
    pdl_enter();
    constexpr int kLanes = D / 8, kGroups = kRotateThreads / kLanes;
    __shared__ float s_dw[kGroups][2][D + 4];
    float w[2][8], dw[2][8] = {};
    load_weights<D>(a, w);
    const int group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    for (int64_t first = (int64_t)blockIdx.x * kGroups; first < a.units; first += (int64_t)gridDim.x * kGroups)
        rotate_unit<T, D, PAIRS, true>(a, first + group, first + group < a.units, w, dw);
    if (a.parts == nullptr) return;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) s_dw[group][s][lane * 8 + e] = dw[s][e];
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kRotateThreads) {
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) sum += s_dw[g][i / D][i % D];
        a.parts[(int64_t)blockIdx.x * 2 * D + i] = sum;
    }
}

// The weights' gradients from the CTAs' parts, always in the same order: 32 columns a CTA, the parts dealt to its warps.
__global__ void __launch_bounds__(1024)
qk_rotate_weights_kernel(const float *parts, int32_t n_parts, int32_t D, float *dq_weight, float *dk_weight) {
    pdl_enter();
    __shared__ double s_sum[32][33];
    const int lane = lane_id(), warp = threadIdx.x >> 5, column = blockIdx.x * kWarp + lane;
    double sum = 0.0;
    for (int32_t p = warp; p < n_parts; p += 32) sum += (double)__ldcg(parts + (int64_t)p * 2 * D + column);
    s_sum[warp][lane] = sum;
    __syncthreads();
    if (warp != 0) return;
    sum = 0.0;
#pragma unroll
    for (int p = 0; p < 32; ++p) sum += s_sum[p][lane];
    float *to = column < D ? dq_weight : dk_weight;
    if (to != nullptr) to[column % D] = (float)sum;
}

template <typename T, int D, bool PAIRS>
static cudaError_t launch_rotate(const RotateArgs &a, bool backward, int grid, cudaStream_t stream) {
    return launch_pdl(backward ? qk_rotate_backward_kernel<T, D, PAIRS> : qk_rotate_kernel<T, D, PAIRS>, grid, kRotateThreads, 0, stream, a);
}

template <typename T>
static cudaError_t launch_rotate_of(const RotateArgs &a, int32_t D, bool pairs, bool backward, int grid, cudaStream_t stream) {
    if (D == 128) return pairs ? launch_rotate<T, 128, true>(a, backward, grid, stream) : launch_rotate<T, 128, false>(a, backward, grid, stream);
    return pairs ? launch_rotate<T, 64, true>(a, backward, grid, stream) : launch_rotate<T, 64, false>(a, backward, grid, stream);
}

static bool rows_ok(const void *p, int64_t stride, int32_t heads, int32_t D, int32_t size) {
    if (heads == 0) return true;
    return p != nullptr && !(reinterpret_cast<uintptr_t>(p) & 15u) && stride >= (int64_t)heads * D && stride * size % 16 == 0;
}

static bool rotate_ok(int32_t dtype, int64_t n, int32_t Hq, int32_t Hk, int32_t D, int32_t rot, int32_t layout, float eps) {
    if (dtype != HORA_DTYPE_F32 && dtype != HORA_DTYPE_BF16 && dtype != HORA_DTYPE_F16) return false;
    if (n < 0 || n > 0x7FFFFFFF || Hq < 0 || Hk < 0 || Hq > 65536 || Hk > 65536 || Hq + Hk < 1 || (D != 64 && D != 128)) return false;
    if (rot < 0 || rot > D || rot % 16 || (layout != HORA_ROTATE_HALVES && layout != HORA_ROTATE_PAIRS)) return false;
    return eps >= 0.f && eps <= 1e30f;
}

static bool tables_ok(const int32_t *positions, const double *inv_freq, int32_t rot, const float *q_weight, const float *k_weight) {
    if (rot > 0 && (positions == nullptr || inv_freq == nullptr)) return false;
    return !(reinterpret_cast<uintptr_t>(inv_freq) & 7u) &&
           !((reinterpret_cast<uintptr_t>(positions) | reinterpret_cast<uintptr_t>(q_weight) | reinterpret_cast<uintptr_t>(k_weight)) & 3u);
}

// How the work is cut: whole tokens while there are enough of them, else a few heads to a unit.
static int units_of(RotateArgs &a, int64_t n, int32_t Hq, int32_t Hk, int32_t D) {
    a.Hq = Hq;
    a.H = Hq + Hk;
    const int64_t most = (a.H + kRotateHeads - 1) / kRotateHeads, want = (kRotateUnits + n - 1) / n;
    const int32_t chunks = (int32_t)(want < most ? want : most);
    a.heads = (a.H + chunks - 1) / chunks;
    a.heads = (a.heads + kRotateHeads - 1) / kRotateHeads * kRotateHeads;
    a.chunks = (a.H + a.heads - 1) / a.heads;
    a.units = n * a.chunks;
    const int64_t groups = kRotateThreads / (D / 8);
    return (int)((a.units + groups - 1) / groups);
}

static hora_status_t launch_rotate_as(const RotateArgs &a, int32_t dtype, int32_t D, int32_t layout, bool backward, int grid, cudaStream_t s) {
    const bool pairs = layout == HORA_ROTATE_PAIRS;
    const cudaError_t e = dtype == HORA_DTYPE_F32    ? launch_rotate_of<float>(a, D, pairs, backward, grid, s)
                          : dtype == HORA_DTYPE_BF16 ? launch_rotate_of<__nv_bfloat16>(a, D, pairs, backward, grid, s)
                                                     : launch_rotate_of<__half>(a, D, pairs, backward, grid, s);
    count_launches(1);
    return cuda_ok(e);
}

}  // namespace hora

extern "C" hora_status_t hora_qk_rotate(const void *q, const void *k, int32_t dtype, int64_t q_row_stride, int64_t k_row_stride, int64_t n_tokens,
                                        int32_t Hq, int32_t Hk, int32_t D, const int32_t *positions, const double *inv_freq, int32_t rot,
                                        int32_t layout, const float *q_weight, const float *k_weight, float eps, void *q_out, void *k_out,
                                        int64_t q_out_row_stride, int64_t k_out_row_stride, void *stream) {
    using namespace hora;
    if (!rotate_ok(dtype, n_tokens, Hq, Hk, D, rot, layout, eps)) return HORA_ERR_INVALID_ARG;
    if (n_tokens == 0) return HORA_OK;
    const int32_t size = dtype_bytes(dtype);
    if (!rows_ok(q, q_row_stride, Hq, D, size) || !rows_ok(k, k_row_stride, Hk, D, size) || !rows_ok(q_out, q_out_row_stride, Hq, D, size) ||
        !rows_ok(k_out, k_out_row_stride, Hk, D, size) || !tables_ok(positions, inv_freq, rot, q_weight, k_weight))
        return HORA_ERR_INVALID_ARG;
    RotateArgs a = {};
    a.x[0] = q; a.x[1] = k;
    a.x_stride[0] = q_row_stride; a.x_stride[1] = k_row_stride;
    a.y[0] = q_out; a.y[1] = k_out;
    a.y_stride[0] = q_out_row_stride; a.y_stride[1] = k_out_row_stride;
    a.w[0] = q_weight; a.w[1] = k_weight;
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.rot = rot;
    a.eps = eps;
    const int grid = units_of(a, n_tokens, Hq, Hk, D);
    return launch_rotate_as(a, dtype, D, layout, false, grid, static_cast<cudaStream_t>(stream));
}

extern "C" size_t hora_qk_rotate_backward_workspace_bytes(int32_t D) {
    return D != 64 && D != 128 ? 0 : (size_t)hora::sm_count() * hora::kRotatePerSm * 2 * D * sizeof(float);
}

extern "C" hora_status_t hora_qk_rotate_backward(const void *dq_out, const void *dk_out, int32_t dtype, int64_t dq_out_row_stride,
                                                 int64_t dk_out_row_stride, const void *q, const void *k, int64_t q_row_stride,
                                                 int64_t k_row_stride, int64_t n_tokens, int32_t Hq, int32_t Hk, int32_t D,
                                                 const int32_t *positions, const double *inv_freq, int32_t rot, int32_t layout,
                                                 const float *q_weight, const float *k_weight, float eps, void *dq, void *dk,
                                                 int64_t dq_row_stride, int64_t dk_row_stride, float *dq_weight, float *dk_weight,
                                                 void *workspace, size_t workspace_bytes, void *stream) {
    using namespace hora;
    if (!rotate_ok(dtype, n_tokens, Hq, Hk, D, rot, layout, eps)) return HORA_ERR_INVALID_ARG;
    if ((dq_weight != nullptr && q_weight == nullptr) || (dk_weight != nullptr && k_weight == nullptr)) return HORA_ERR_INVALID_ARG;
    const int32_t size = dtype_bytes(dtype);
    if (n_tokens > 0) {
        if (!rows_ok(dq_out, dq_out_row_stride, Hq, D, size) || !rows_ok(dk_out, dk_out_row_stride, Hk, D, size) ||
            !rows_ok(dq, dq_row_stride, Hq, D, size) || !rows_ok(dk, dk_row_stride, Hk, D, size))
            return HORA_ERR_INVALID_ARG;
        if ((q_weight != nullptr && !rows_ok(q, q_row_stride, Hq, D, size)) || (k_weight != nullptr && !rows_ok(k, k_row_stride, Hk, D, size)) ||
            !tables_ok(positions, inv_freq, rot, q_weight, k_weight) ||
            ((reinterpret_cast<uintptr_t>(dq_weight) | reinterpret_cast<uintptr_t>(dk_weight)) & 3u))
            return HORA_ERR_INVALID_ARG;
    }
    const bool weights = dq_weight != nullptr || dk_weight != nullptr;
    if (weights && (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < hora_qk_rotate_backward_workspace_bytes(D)))
        return HORA_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int grid = 0;
    if (n_tokens > 0) {
        RotateArgs a = {};
        a.x[0] = q; a.x[1] = k;
        a.x_stride[0] = q_row_stride; a.x_stride[1] = k_row_stride;
        a.dy[0] = dq_out; a.dy[1] = dk_out;
        a.dy_stride[0] = dq_out_row_stride; a.dy_stride[1] = dk_out_row_stride;
        a.y[0] = dq; a.y[1] = dk;
        a.y_stride[0] = dq_row_stride; a.y_stride[1] = dk_row_stride;
        a.w[0] = q_weight; a.w[1] = k_weight;
        a.positions = positions;
        a.inv_freq = inv_freq;
        a.rot = rot;
        a.eps = eps;
        a.parts = weights ? static_cast<float *>(workspace) : nullptr;
        grid = clamp_grid(units_of(a, n_tokens, Hq, Hk, D), kRotatePerSm);
        const hora_status_t rc = launch_rotate_as(a, dtype, D, layout, true, grid, s);
        if (rc != HORA_OK) return rc;
    }
    if (!weights) return HORA_OK;
    const cudaError_t e = launch_pdl(qk_rotate_weights_kernel, 2 * D / kWarp, 1024, 0, s, static_cast<const float *>(workspace), (int32_t)grid, D, dq_weight, dk_weight);
    count_launches(1);
    return cuda_ok(e);
}
