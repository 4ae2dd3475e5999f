// hora_group_attention, the kernel for wide items: many query rows to a key, as the prompt's keys of a large group have.
//
// S = Q K^T and O += P V on the tensor cores' own memory: tcgen05.mma takes 128 rows at a time, S (128 x 128) and O
// (128 x D) are accumulated in tensor memory, the weights P replace the scores there and are the left operand of the second
// product.  A CTA is a stream and holds an SM: two halves of 128 rows, each with four warps that do its softmax, one thread to a row,
// share the keys and values that one warp brings in by TMA; one thread issues all products.  While one half does
// its softmax the tensor cores work for the other.  An item with no more than 128 rows gives both halves the same rows and deals
// them the key tiles in turn: two partials, joined like all others.
//   Keys (K-major) and queries lie in shared memory in rows of 128 bytes with the 128-byte swizzle, values as they come are the
// right operand with the head's dimension contiguous: nothing is transposed.
//   The reference score of a row is raised only when a tile's maximum exceeds it by 2^8 (weights up to 256 are as exact as
// weights up to 1 in floating point), so O is hardly ever rescaled.
//   Keys beyond the length are not fetched; the product stops at the last sixteen that hold one, and what is beyond the length
// among those is cleared in shared memory first (0 * NaN is not 0).
//   Every wait has a limit; a wait that reaches it makes the CTA give up and report HORA_ERR_INTERNAL.
#include <cuda.h>

#include <type_traits>

#include "hora_group_attention.cuh"

namespace hora {

constexpr int kWideThreads = 384;                        // two halves of four warps; one for TMA, one for the products, one for the list of pieces, a spare one
constexpr int kTmaWarp = 8, kMmaWarp = 9, kListWarp = 10;
constexpr int kPieceBatch = 32;                          // pieces listed at a time
// Registers: launched with 168 a thread (three warps share a scheduler's 16384); the softmax warps, which hold 128 scores each thread, take
// what the others leave: 2 * 224 + 56 = 3 * 168.
constexpr int kSoftmaxRegs = 224, kOtherRegs = 56;
constexpr uint32_t kWaitTries = 4000000;                 // of at least a microsecond each unless the barrier is passed

template <int D>
struct WideSmem {
    static constexpr int kQBytes = kWideHalf * D * 2;
    static constexpr int kStageBytes = kWideKeys * D * 2;             // keys or values of a step
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int kQ = 0;                                      // [2][D / 64][128][128 bytes]
    static constexpr int kRing = 2 * kQBytes;                         // [stages][D / 64][128][128 bytes]
    static constexpr int kBars = kRing + kStages * kStageBytes;
    static constexpr int kBytes = kBars + 256 + 1024;                 // and room to begin on a multiple of 1024
};

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Waits for the phase of the given parity to complete; false when the limit is reached or another wait of the CTA has failed.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int32_t *failed) {
    for (uint32_t i = 0; i < kWaitTries; ++i) {
        uint32_t done;
        asm volatile(
            "{\n.reg .pred p;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
            "selp.b32 %0, 1, 0, p;\n}"
            : "=r"(done)
            : "r"(bar), "r"(parity), "r"(1000u)
            : "memory");
        if (done) return true;
        if (*failed) return false;
    }
    *failed = 1;
    return false;
}

__device__ __forceinline__ void tma_box(uint32_t to, const CUtensorMap *map, int32_t x, int32_t y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map),
                 "r"(x), "r"(y), "r"(bar)
                 : "memory");
}

// Operand in shared memory, 128-byte swizzle.  `lead`: distance between blocks of 64 elements along the contiguous
// direction (used when that is the direction of the rows or columns of the product), groups of eight lie 1024 bytes apart.
// The low word; the high one is the same for all.
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t lead) { return ((at & 0x3FFFFu) >> 4) | ((lead >> 4) << 16); }
constexpr uint32_t kOperandHigh = (1024u >> 4) | (1u << 14) | (2u << 29);

__device__ __forceinline__ void mma_smem(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 da, db;\nmov.b64 da, {%1, %5};\nmov.b64 db, {%2, %5};\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(kOperandHigh)
        : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 db;\nmov.b64 db, {%2, %5};\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(kOperandHigh)
        : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of tensor memory, the warp's 32 lanes: one row of them to a thread.
__device__ __forceinline__ void tmem_load(uint32_t at, float (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
          "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]),
          "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]),
          "=f"(r[30]), "=f"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
        "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
        "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(at)
        : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A piece as the warps of its CTA need it.
struct WidePiece {
    const int32_t *pages;
    int32_t first, seq_rows, len;                        // of the sequence
    int32_t h, row0, rows, key0, n;                      // head, rows of the item, first key, key tiles
    bool prompt, continued;
    bool both;                                           // both halves take every tile (their rows differ)

    // key tiles of a half, and which its k-th is
    __device__ __forceinline__ int32_t count(int half) const { return both ? n : (n + 1 - half) >> 1; }
    __device__ __forceinline__ int32_t key(int half, int32_t k) const { return key0 + (both ? k : 2 * k + half) * kWideKeys; }
};

// What the warps of a CTA share beside the tiles.
struct WideBars {
    uint32_t full, empty, scores, weights, queries, output;          // arrays of 8-byte barriers: [stages] x 2, [2] x 4
};

// O of a warp's rows, times f.
template <int D>
__device__ __forceinline__ void scale_output(uint32_t t_o, float f) {
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
        float o[32];
        uint32_t y[32];
        tmem_load(t_o + b * 32, o);
        tmem_load_wait();
#pragma unroll
        for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(o[e] * f);
        tmem_store(t_o + b * 32, y);
    }
}

template <typename Q, int D>
__global__ void __launch_bounds__(kWideThreads, 1)
attention_wide_kernel(const AttnArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    pdl_enter();
    using Smem = WideSmem<D>;
    constexpr int kStages = Smem::kStages, kParts = D / 64;
    extern __shared__ uint8_t s_raw[];
    __shared__ int32_t s_failed;
    __shared__ uint32_t s_tmem;
    __shared__ WidePiece s_piece[kPieceBatch];
    __shared__ int32_t s_pieces;
    const uint32_t base = (smem_at(s_raw) + 1023u) & ~1023u;
    const WideBars bars = {base + Smem::kBars, base + Smem::kBars + 8 * kStages, base + Smem::kBars + 16 * kStages,
                           base + Smem::kBars + 16 * kStages + 16, base + Smem::kBars + 16 * kStages + 32, base + Smem::kBars + 16 * kStages + 48};
    const int warp = threadIdx.x >> 5, lane = lane_id();
    bool bad = false;
    if ((int64_t)blockIdx.x * steps_per_stream<true>(a) >= __ldg(a.start[1] + a.N + a.R)) return;       // nothing on this stream

    if (threadIdx.x == 0) {
        s_failed = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(bars.full + 8 * s, 1);
            bar_init(bars.empty + 8 * s, 1);
        }
        for (int h = 0; h < 2; ++h) {
            bar_init(bars.scores + 8 * h, 1);
            bar_init(bars.weights + 8 * h, kWideHalf);
            bar_init(bars.queries + 8 * h, kWideHalf);
            bar_init(bars.output + 8 * h, 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_at(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = s_tmem;                        // columns: S of the halves, 128 each, then O, D each
    volatile int32_t *failed = &s_failed;

    // All warps go through the stream's pieces in batches: one warp lists a batch, the others work through it.  Returns how many there are.
    auto next_batch = [&]() {
        __syncthreads();
        return s_failed ? 0 : s_pieces;
    };
    if (warp >= kTmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp >= kListWarp) {
            Pieces<true> pieces(a, blockIdx.x, bad);
            int32_t n = 1;
            while (n > 0) {
                n = 0;
                Piece w;
                while (warp == kListWarp && n < kPieceBatch && pieces.next(a, w, bad)) {
                    if (lane == 0) {
                        WidePiece &p = s_piece[n];
                        p.pages = w.pages;
                        p.first = pieces.s.first;
                        p.seq_rows = pieces.s.rows;
                        p.len = pieces.s.len;
                        p.h = w.h;
                        p.row0 = w.row0;
                        p.rows = w.rows;
                        p.key0 = w.step0 * kWideKeys;
                        p.n = w.step1 - w.step0;
                        p.prompt = w.prompt;
                        p.continued = w.step0 > 0;
                        p.both = w.rows > kWideHalf;
                    }
                    ++n;
                }
                if (warp == kListWarp && lane == 0) s_pieces = n;
                n = next_batch();
                __syncthreads();                             // the batch has been worked through
            }
        } else if (warp == kTmaWarp) {
            // ---- keys and values: the stages in the order of their first use
            int32_t pos = 0;                                 // stages handed out so far
            const int page = 1 << a.page_shift;
            const int lane_box = lane / kParts, lane_part = lane % kParts;
            bool ok = true;
            auto bring = [&](const CUtensorMap *map, const WidePiece &p, int32_t key0) {
                const int32_t boxes = (min(kWideKeys, p.len - key0) + page - 1) >> a.page_shift;
                const int stage = pos % kStages;
                int32_t id = 0;
                if (lane_box < boxes) id = __ldg(p.pages + (key0 >> a.page_shift) + lane_box);
                if (id < 0 || id >= a.n_pages) { bad = true; id = 0; }
                if (pos >= kStages) ok = bar_wait(bars.empty + 8 * stage, (pos / kStages + 1) & 1, failed);
                ok = __all_sync(kFull, ok);
                if (!ok) return;
                if (lane == 0) bar_expect(bars.full + 8 * stage, boxes * page * D * 2);
                __syncwarp();
                if (lane_box < boxes)
                    tma_box(base + Smem::kRing + stage * Smem::kStageBytes + lane_part * (kWideKeys * 128) + lane_box * page * 128, map, lane_part * 64,
                            (int32_t)(((int64_t)id * a.Hkv + p.h) << a.page_shift), bars.full + 8 * stage);
                ++pos;
            };
            while (const int32_t listed = next_batch()) {
                for (int32_t at = 0; at < listed && ok; ++at) {
                    const WidePiece &p = s_piece[at];
                    const int32_t n = p.count(0), halves = p.both ? 1 : 2;
                    for (int32_t it = 0; it <= n && ok; ++it)
                        for (int half = 0; half < halves && ok; ++half) {
                            if (it >= 1 && it - 1 < p.count(half)) bring(&v_map, p, p.key(half, it - 1));
                            if (it < p.count(half) && ok) bring(&k_map, p, p.key(half, it));
                        }
                }
                // the CTA may not end while copies are on their way to it: every stage's copy is waited for by its use, unless
                // the CTA has given up
                if (!ok)
                    for (int32_t x = max(0, pos - kStages); x < pos; ++x) {
                        int32_t never = 0;
                        bar_wait(bars.full + 8 * (x % kStages), (x / kStages) & 1, &never);
                    }
                __syncthreads();
            }
            __syncthreads();
        } else if (warp == kMmaWarp) {
            // ---- products
            constexpr uint32_t kType = std::is_same<Q, __nv_bfloat16>::value ? 1u : 0u;
            constexpr uint32_t kIdescS = (1u << 4) | (kType << 7) | (kType << 10) | ((kWideKeys / 8) << 17) | ((kWideHalf / 16) << 24);
            constexpr uint32_t kIdescO = (1u << 4) | (kType << 7) | (kType << 10) | (1u << 16) | ((D / 8) << 17) | ((kWideHalf / 16) << 24);
            int32_t pos = 0, k_pos = 0, v_pos = 0;
            uint32_t n_weights[2] = {0, 0}, n_queries[2] = {0, 0};
            bool ok = true;
            while (const int32_t listed = next_batch()) {
                for (int32_t at = 0; at < listed && ok; ++at) {
                    const WidePiece &p = s_piece[at];
                    const int32_t n0 = p.count(0);
                    for (int32_t it = 0; it <= n0 && ok; ++it) {
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            if (!ok) break;
                            const int32_t n = p.count(half);
                            const bool first_use = !p.both || half == 0, last_use = !p.both || half == 1;
                            if (it >= 1 && it - 1 < n) {
                                if (first_use) v_pos = pos++;
                                const int stage = v_pos % kStages;
                                ok = bar_wait(bars.weights + 8 * half, n_weights[half]++ & 1, failed) &&
                                     bar_wait(bars.full + 8 * stage, (v_pos / kStages) & 1, failed);
                                if (!ok) break;
                                fence_after();
                                const int32_t groups = (min(kWideKeys, p.len - p.key(half, it - 1)) + 15) >> 4;
                                if (lane == 0) {
                                    const uint32_t v = operand(base + Smem::kRing + stage * Smem::kStageBytes, kWideKeys * 128);
#pragma unroll
                                    for (int g = 0; g < kWideKeys / 16; ++g)
                                        if (g < groups)
                                            mma_tmem(tmem + 256 + half * D, tmem + half * 128 + g * 8, v + g * (2048 >> 4), kIdescO, it > 1 || g > 0);
                                    if (last_use) mma_commit(bars.empty + 8 * stage);
                                    if (it == n) mma_commit(bars.output + 8 * half);
                                }
                                __syncwarp();
                            }
                            if (it < n) {
                                if (first_use) k_pos = pos++;
                                const int stage = k_pos % kStages;
                                if (it == 0) ok = bar_wait(bars.queries + 8 * half, n_queries[half]++ & 1, failed);
                                ok = ok && bar_wait(bars.full + 8 * stage, (k_pos / kStages) & 1, failed);
                                if (!ok) break;
                                fence_after();
                                if (lane == 0) {
                                    const uint32_t q = operand(base + Smem::kQ + half * Smem::kQBytes, 16);
                                    const uint32_t k = operand(base + Smem::kRing + stage * Smem::kStageBytes, 16);
#pragma unroll
                                    for (int x = 0; x < D / 16; ++x) {
                                        const uint32_t off = ((x >> 2) * (kWideKeys * 128) + (x & 3) * 32) >> 4;
                                        mma_smem(tmem + half * 128, q + off, k + off, kIdescS, x > 0);
                                    }
                                    mma_commit(bars.scores + 8 * half);
                                    if (last_use) mma_commit(bars.empty + 8 * stage);
                                }
                                __syncwarp();
                            }
                        }
                    }
                }
                __syncthreads();
            }
            __syncthreads();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // ---- softmax: thread `row` of a half has row `row` of its scores
        const int half = warp >> 2, row = threadIdx.x & (kWideHalf - 1);
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);           // this warp's 32 lanes of tensor memory
        const uint32_t t_s = lanes + half * 128, t_o = lanes + 256 + half * D;
        uint32_t n_scores = 0, n_output = 0;
        int32_t pos = 0;                                 // stages of all pieces before this one
        bool ok = true;
        while (const int32_t listed = next_batch()) {
            for (int32_t at = 0; at < listed; ++at) {
                const WidePiece &p = s_piece[at];
                const int32_t n = p.count(half);
                const int32_t x = (p.both ? half * kWideHalf : 0) + row;      // row of the item
                QueryRow qr = {-1, 0};
                if (x < p.rows) qr = query_row(a, p.first, p.seq_rows, p.len, p.prompt, p.h, p.row0 + x);
                const bool warp_has_rows = __any_sync(kFull, qr.out >= 0);
                float m = -INFINITY, l = 0.f;
                if (n > 0) {
                    // queries into shared memory; the products that read the last ones are done (their output was waited for)
                    if (warp_has_rows) {
                        const Q *__restrict__ q = static_cast<const Q *>(a.q) + (qr.out >= 0 ? qr.out / a.Hq * a.q_row_stride + qr.out % a.Hq * D : 0);
                        const uint32_t to = base + Smem::kQ + half * Smem::kQBytes + row * 128;
#pragma unroll
                        for (int c = 0; c < D / 8; ++c) {
                            const uint4 v = qr.out >= 0 ? __ldg(reinterpret_cast<const uint4 *>(q) + c) : make_uint4(0, 0, 0, 0);
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to + (c >> 3) * (kWideHalf * 128) + (((c & 7) ^ (row & 7)) << 4)),
                                         "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                                         : "memory");
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    bar_arrive(bars.queries + 8 * half);
                    for (int32_t k = 0; k < n; ++k) {
                        const int32_t key0 = p.key(half, k);
                        ok = ok && bar_wait(bars.scores + 8 * half, n_scores++ & 1, failed);
                        ok = __all_sync(kFull, ok);
                        if (!ok) break;
                        fence_after();
                        if (warp_has_rows) {
                            float s[4][32];
#pragma unroll
                            for (int b = 0; b < 4; ++b) tmem_load(t_s + b * 32, s[b]);
                            tmem_load_wait();
                            if (key0 + kWideKeys > qr.limit) {
#pragma unroll
                                for (int b = 0; b < 4; ++b)
#pragma unroll
                                    for (int e = 0; e < 32; ++e)
                                        if (key0 + b * 32 + e >= qr.limit) s[b][e] = -INFINITY;
                            }
                            float top = -INFINITY;
#pragma unroll
                            for (int b = 0; b < 4; ++b)
#pragma unroll
                                for (int e = 0; e < 32; ++e) top = fmaxf(top, s[b][e]);
                            top *= a.scale_log2;
                            if (k == 0) {
                                m = top;
                            } else if (__any_sync(kFull, top > m + 8.f)) {
                                const float up = fmaxf(m, top), f = up == -INFINITY ? 1.f : exp2_fast(m - up);
                                l *= f;
                                m = up;
                                scale_output<D>(t_o, f);
                            }
                            // where no key has been seen the reference is -infinity and every weight has to come out as 0
                            const float z = m == -INFINITY ? 0.f : m;
#pragma unroll
                            for (int b = 0; b < 2; ++b) {
                                uint32_t w[32];
#pragma unroll
                                for (int e = 0; e < 32; ++e) {
                                    const float p0 = exp2_fast(fmaf(s[2 * b + (e >> 4)][(2 * e) & 31], a.scale_log2, -z));
                                    const float p1 = exp2_fast(fmaf(s[2 * b + (e >> 4)][(2 * e + 1) & 31], a.scale_log2, -z));
                                    l += p0 + p1;
                                    w[e] = pack2(p0, p1, Q());
                                }
                                tmem_store(t_s + b * 32, w);
                            }
                            tmem_store_wait();
                        }
                        // the last tile's values beyond the length, among the sixteen keys that the product reads last
                        const int32_t keys = p.len - key0;
                        if (keys < kWideKeys && (keys & 15) != 0 && !(p.both && half == 1)) {
                            const int32_t last = pos + 2 * p.n - 1;           // the piece's last stage holds them
                            const uint32_t stage = base + Smem::kRing + last % kStages * Smem::kStageBytes;
                            ok = bar_wait(bars.full + 8 * (last % kStages), (last / kStages) & 1, failed);
                            const int32_t clear = ((keys + 15) & ~15) - keys;
                            if (ok)
                                for (int32_t c = row; c < clear * (D / 8); c += kWideHalf) {
                                    const int32_t r = keys + c / (D / 8), chunk = c % (D / 8);
                                    asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(stage + (chunk >> 3) * (kWideKeys * 128) + r * 128 + (chunk & 7) * 16),
                                                 "r"(0)
                                                 : "memory");
                                }
                            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        }
                        fence_before();
                        bar_arrive(bars.weights + 8 * half);
                    }
                    ok = ok && bar_wait(bars.output + 8 * half, n_output++ & 1, failed);
                    ok = __all_sync(kFull, ok);
                    if (!ok) break;
                    fence_after();
                }
                pos += 2 * p.n;
                if (!warp_has_rows) continue;
                // the partial
                const int64_t rows_all = (int64_t)a.R * a.T * a.Hq;
                const int64_t place = p.continued ? (int64_t)blockIdx.x * kWideRows + half * kWideHalf + row
                                                  : (int64_t)((p.prompt ? kPromptPart : kOwnPart) + (!p.both && half ? kSecondHalf : 0)) * rows_all + qr.out;
                float *__restrict__ po = (p.continued ? a.cont_o[1] : a.main_o) + place * D;
                if (n > 0) {
#pragma unroll
                    for (int b = 0; b < D / 32; ++b) {
                        float o[32];
                        tmem_load(t_o + b * 32, o);
                        tmem_load_wait();
                        if (qr.out >= 0) {
#pragma unroll
                            for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4 *>(po + b * 32 + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                        }
                    }
                }
                if (qr.out >= 0) *reinterpret_cast<float2 *>((p.continued ? a.cont_ml[1] : a.main_ml) + place * 2) = make_float2(m, l);
                fence_before();                          // the next item's products may overwrite O: its weights come after this
            }
            __syncthreads();
        }
        __syncthreads();
    }
    if (bad) raise_status(a.status, HORA_ERR_INVALID_VALUE);
    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && s_failed) raise_status(a.status, HORA_ERR_INTERNAL);
    if (warp == 0) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// One pool as a matrix of [pages * heads * page_size] rows of D elements, fetched 64 elements of one page's rows at a time.
static bool pool_map(CUtensorMap *map, const void *pool, int32_t dtype, int64_t rows, int32_t D, int32_t page) {
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    if (encode == nullptr) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)D * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)page}, steps[2] = {1, 1};
    return encode(map, dtype == HORA_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(pool), dims,
                  strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename Q, int D>
static hora_status_t launch_wide(const AttnArgs &a, int32_t dtype, cudaStream_t stream) {
    CUtensorMap k, v;
    const int64_t rows = (a.n_pages * a.Hkv) << a.page_shift;
    if (!pool_map(&k, a.k_cache, dtype, rows, D, 1 << a.page_shift) || !pool_map(&v, a.v_cache, dtype, rows, D, 1 << a.page_shift)) return HORA_ERR_CUDA;
    constexpr int kSmem = WideSmem<D>::kBytes;
    cudaError_t e = cudaFuncSetAttribute(attention_wide_kernel<Q, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e == cudaSuccess) e = launch_pdl(attention_wide_kernel<Q, D>, a.n_wide, kWideThreads, kSmem, stream, a, k, v);
    count_launches(1);
    return cuda_ok(e);
}

hora_status_t launch_attention_wide(const AttnArgs &a, int32_t q_dtype, int32_t D, cudaStream_t stream) {
    if (q_dtype == HORA_DTYPE_BF16) return D == 64 ? launch_wide<__nv_bfloat16, 64>(a, q_dtype, stream) : launch_wide<__nv_bfloat16, 128>(a, q_dtype, stream);
    return D == 64 ? launch_wide<__half, 64>(a, q_dtype, stream) : launch_wide<__half, 128>(a, q_dtype, stream);
}

}  // namespace hora
