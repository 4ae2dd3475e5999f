// hora_group_attention: the kernel.  One CTA of twelve warps to an SM: together they are a stream of the wide line (products on
// tcgen05), then each of them is a stream of the narrow line.  One launch for both, so that no SM waits for the slowest
// of the others in between.
#include <atomic>

#define HORA_FILE_ID 6
#include "hora_group_attention_narrow.cuh"
#include "hora_group_attention_wide.cuh"

HORA_CHECKED_REGISTER()

namespace hora {

template <bool F8, int D>
constexpr int attention_smem() {
    constexpr int kRings = kNarrowPerSm * Stage<F8, D>::kWarpBytes, kWide = WideSmem<D>::kSmall + (int)sizeof(WideShared);
    return F8 || kRings > kWide ? kRings : kWide;
}

template <typename Q, int D, int NT>
__global__ void __launch_bounds__(kAttnThreads, 1)
attention_kernel(const AttnArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    pdl_enter();
    if (smem_at(s_attention) & 1023u) {
        raise_status(a.status, HORA_ERR_INTERNAL);
        return;
    }
    wide_stream<Q, D>(a, k_map, v_map, s_attention);
    const int warp = threadIdx.x >> 5;
    narrow_stream<Q, false, D, NT>(a, blockIdx.x * kNarrowPerSm + warp, smem_at(s_attention) + warp * Stage<false, D>::kWarpBytes);
}

// An e4m3 cache: every item is narrow.
template <typename Q, int D, int NT>
__global__ void __launch_bounds__(kAttnThreads, 1)
attention_e4m3_kernel(const AttnArgs a) {
    pdl_enter();
    const int warp = threadIdx.x >> 5;
    narrow_stream<Q, true, D, NT>(a, blockIdx.x * kNarrowPerSm + warp, smem_at(s_attention) + warp * Stage<true, D>::kWarpBytes);
}

// One pool as a matrix of [pages * heads * page_size] rows of D elements, fetched 64 elements of one page's rows at a time.
static bool pool_map(CUtensorMap *map, const void *pool, int32_t dtype, int64_t rows, int32_t D, int32_t page) {
    const TensorMapEncode encode = tensor_map_encode();
    if (encode == nullptr) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)D * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)page}, steps[2] = {1, 1};
    return encode(map, dtype == HORA_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(pool), dims,
                  strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename Q, int D, int NT>
static hora_status_t launch(const AttnArgs &a, int32_t q_dtype, bool f8, cudaStream_t stream) {
    cudaError_t e;
    if (f8) {
        constexpr int kSmem = attention_smem<true, D>();
        static std::atomic<uint64_t> devices{0};
        e = allow_shared(reinterpret_cast<const void *>(attention_e4m3_kernel<Q, D, NT>), kSmem, devices);
        if (e == cudaSuccess) e = launch_pdl(attention_e4m3_kernel<Q, D, NT>, a.n_sm, kAttnThreads, kSmem, stream, a);
    } else {
        CUtensorMap k, v;
        const int64_t rows = (a.n_pages * a.Hkv) << a.page_shift;
        if (!pool_map(&k, a.k_cache, q_dtype, rows, D, 1 << a.page_shift) || !pool_map(&v, a.v_cache, q_dtype, rows, D, 1 << a.page_shift)) return HORA_ERR_CUDA;
        constexpr int kSmem = attention_smem<false, D>();
        static std::atomic<uint64_t> devices{0};
        e = allow_shared(reinterpret_cast<const void *>(attention_kernel<Q, D, NT>), kSmem, devices);
        if (e == cudaSuccess) e = launch_pdl(attention_kernel<Q, D, NT>, a.n_sm, kAttnThreads, kSmem, stream, a, k, v);
    }
    count_launches(1);
    return cuda_ok(e);
}

template <typename Q>
static hora_status_t launch_for(const AttnArgs &a, int32_t q_dtype, bool f8, int32_t D, cudaStream_t stream) {
    const int nt = a.narrow_rows / 8;
    if (D == 128) return nt == 1 ? launch<Q, 128, 1>(a, q_dtype, f8, stream) : launch<Q, 128, 2>(a, q_dtype, f8, stream);
    return nt == 1 ? launch<Q, 64, 1>(a, q_dtype, f8, stream) : nt == 2 ? launch<Q, 64, 2>(a, q_dtype, f8, stream) : launch<Q, 64, 3>(a, q_dtype, f8, stream);
}

hora_status_t launch_attention_main(const AttnArgs &a, int32_t q_dtype, int32_t cache_dtype, int32_t D, cudaStream_t stream) {
    const bool f8 = cache_dtype == HORA_DTYPE_E4M3;
    return q_dtype == HORA_DTYPE_BF16 ? launch_for<__nv_bfloat16>(a, q_dtype, f8, D, stream) : launch_for<__half>(a, q_dtype, f8, D, stream);
}

}  // namespace hora
