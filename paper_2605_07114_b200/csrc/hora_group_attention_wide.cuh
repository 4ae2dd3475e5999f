// hora_group_attention: wide items: many query rows to a key, as the prompt's keys of a large group have.
//
// S = Q K^T and O += P V on the tensor cores' own memory: tcgen05.mma takes 128 rows at a time, S (128 x 64, twice) and O
// (128 x D) are accumulated in tensor memory, the weights P replace the scores there and are the left operand of the second
// product.  A CTA is a stream and holds an SM: two halves of 128 rows share the keys and values that one warp brings in by TMA.
// Each half has one warp that issues its products and four that do its softmax, one thread to a row.  The chain scores -> maximum ->
// weights -> product takes much longer than its products, so four of them are under way at any time: a step's 128 keys
// make two tiles, and while a half's softmax works on one the tensor cores compute the scores of the next.  An item with no more
// than 128 rows gives both halves the same rows and deals them the steps in turn: two partials, joined like all others.
//   Keys (K-major) and queries lie in shared memory in rows of 128 bytes with the 128-byte swizzle, values as they come are the
// right operand with the head's dimension contiguous: nothing is transposed.
//   The reference score of a row is raised only when a tile's maximum exceeds it by 2^8 (weights up to 256 are as exact as
// weights up to 1 in floating point), so O is hardly ever rescaled.
//   Keys beyond the length are not fetched; the product stops at the last sixteen that hold one, and what is beyond the length
// among those is cleared in shared memory first (0 * NaN is not 0).
//   What bounds it: the chain, where both halves have rows of their own (2.3 us a step of 256 rows and 128 keys of D = 128, 825 TFLOP/s
// over 103485 keys and 512 rows; with an eighth of the bytes a step takes as long); HBM for items of one half (1.6 us a step of
// 64 KiB, 0.93 of the copy rate).  A quarter of the exponentials by products: 384 us in place of 392 for 1024 queries of 64 heads.
//   Every wait has a limit; a wait that reaches it makes the CTA give up and report HORA_ERR_INTERNAL.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "hora_group_attention_narrow.cuh"

namespace hora {

constexpr int kSoftmaxWarps = 8, kHalfThreads = kSoftmaxWarps / 2 * kWarp;
constexpr int kTmaWarp = kSoftmaxWarps, kMmaWarp = kTmaWarp + 1, kListWarp = kMmaWarp + 2;        // one for TMA, one a half for the products, one to list the pieces
static_assert((kListWarp + 1) * kWarp == kAttnThreads, "every warp has a role");
constexpr int kTileKeys = 64;
constexpr int kPieceBatch = 16;                          // pieces listed at a time
constexpr uint32_t kWaitTries = 4000000;                 // a fraction of a second and more; what is waited for takes microseconds

template <int D>
struct WideSmem {
    static constexpr int kQBytes = kWideHalf * D * 2;
    static constexpr int kStageBytes = kWideKeys * D * 2;             // keys or values of a step
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int kQ = 0;                                      // [2][D / 64][128][128 bytes]
    static constexpr int kRing = 2 * kQBytes;                         // [stages][D / 64][128][128 bytes]
    static constexpr int kSmall = kRing + kStages * kStageBytes;       // WideShared
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
    (void)HORA_IN(-1, 1);
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
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0;
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
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
          "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
        : "r"(at));
}
__device__ __forceinline__ void tmem_store8(uint32_t at, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
                 "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const float (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"f"(r[0]), "f"(r[1]),
        "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "f"(r[8]), "f"(r[9]), "f"(r[10]), "f"(r[11]), "f"(r[12]), "f"(r[13]),
        "f"(r[14]), "f"(r[15]), "r"(at)
        : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A piece as the warps of its CTA need it.
struct WidePiece {
    const int32_t *pages;
    int32_t first, seq_rows, len;                        // of the sequence
    int32_t h, row0, rows, key0, n;                      // head, rows of the item, first key, key tiles
    bool prompt, continued;
    bool both;                                           // both halves take every tile (their rows differ)

    // steps of a half, the first key of its k-th, and the tiles of all of them
    __device__ __forceinline__ int32_t count(int half) const { return both ? n : (n + 1 - half) >> 1; }
    __device__ __forceinline__ int32_t key(int half, int32_t k) const { return key0 + (both ? k : 2 * k + half) * kWideKeys; }
    __device__ __forceinline__ int32_t tiles(int half) const {
        const int32_t k = count(half);
        return k == 0 ? 0 : 2 * k - (len - key(half, k - 1) <= kTileKeys ? 1 : 0);
    }
};

// What the warps of a CTA share beside the tiles.
struct WideBars {
    uint32_t full, empty, scores, weights, queries, product, output;           // 8-byte barriers: [stages] x 2, [half][tile & 1] x 2, [half] x 3
};

__device__ __forceinline__ void store16(uint32_t at, const uint4 &v) {
    if (!HORA_IN(in_shared(at, 16), 1)) return;
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 load16(uint32_t at) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (!HORA_IN(in_shared(at, 16), 1)) return v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// Two fp32 operations an instruction.
__device__ __forceinline__ uint64_t two(float2 x) { return (uint64_t)__float_as_uint(x.y) << 32 | __float_as_uint(x.x); }
__device__ __forceinline__ float2 two(uint64_t x) { return make_float2(__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32))); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(two(a)), "l"(two(b)), "l"(two(c)));
    return two(d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(two(a)), "l"(two(b)));
    return two(d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(two(a)), "l"(two(b)));
    return two(d);
}
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// 2^x by multiplications, for x <= 8: the special function unit takes 8 cycles a warp, as long as the tensor cores need for its
// share of the products, so a quarter of the exponentials is computed beside it.  2^x = 2^n 2^f, n = round(x), |f| <= 1/2;
// 2^f by the polynomial of degree 5 with the least largest relative error (7.5e-8, 2.0e-7 with fp32 rounding; fitted by iterated
// weighted least squares), times 2^n, whose exponent comes from the low bits of the rounding.  Below 2^-126.5, for the -infinity of a hidden
// key too, 2^n is 0 and so is the result, as the special function unit has it; NaN stays NaN.
__device__ __forceinline__ float2 exp2_by_products(float2 x) {
    x = make_float2(max_or_nan(x.x, -127.f), max_or_nan(x.y, -127.f));
    const float2 big = make_float2(12582912.f, 12582912.f), t = add2(x, big);      // 1.5 * 2^23: the low bits of t are n
    const float2 f = fma2(add2(t, make_float2(-12582912.f, -12582912.f)), make_float2(-1.f, -1.f), x);
    float2 p = make_float2(1.3276471519402e-3f, 1.3276471519402e-3f);
    p = fma2(p, f, make_float2(9.6755413306768e-3f, 9.6755413306768e-3f));
    p = fma2(p, f, make_float2(5.5507132749614e-2f, 5.5507132749614e-2f));
    p = fma2(p, f, make_float2(2.4022119723934e-1f, 2.4022119723934e-1f));
    p = fma2(p, f, make_float2(6.9314696706386e-1f, 6.9314696706386e-1f));
    p = fma2(p, f, make_float2(1.0000000716547f, 1.0000000716547f));
    return mul2(p, make_float2(__uint_as_float((__float_as_uint(t.x) << 23) + 0x3F800000u), __uint_as_float((__float_as_uint(t.y) << 23) + 0x3F800000u)));
}

// O of a warp's rows, times f; few columns at a time, since the scores are in registers meanwhile.
template <int D>
__device__ __forceinline__ void scale_output(uint32_t t_o, float f) {
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

struct WideShared {
    uint64_t bars[40];
    WidePiece piece[kPieceBatch];
    int32_t pieces, failed;
    int32_t issued;                                      // copies begun so far
    uint32_t tmem;
};

// Waits for the copy into a stage, number `pos` of all.  A warp may come here many stages after the last one that it waited for
// (the others were the other half's), and a barrier only tells two neighbouring phases apart: the count of the copies begun says that
// the stage's copy before this one is over.
template <int STAGES>
__device__ __forceinline__ bool wait_for_copy(const WideShared &sh, const WideBars &bars, int32_t pos, volatile int32_t *failed) {
    const volatile int32_t *issued = &sh.issued;
    for (uint32_t i = 0; *issued <= pos; ++i)
        if (*failed || i >= kWaitTries * 8) {
            *failed = 1;
            (void)HORA_IN(-1, 1);
            return false;
        }
    return bar_wait(bars.full + 8 * (pos % STAGES), (pos / STAGES) & 1, failed);
}

// Clears the values beyond the last of a tile's `keys` keys, among the sixteen that the product reads last: they may be anything,
// and 0 * NaN is not 0.  The tile is the last (number `tile` of its step) of the piece, whose last stage, number `last`, holds its
// values; a half whose tiles end before that has nothing to clear.  All threads of a half; where both halves read the stage
// both do it, since either may be the first to need it.
template <int D>
__device__ __forceinline__ bool clear_values(const WideShared &sh, const WideBars &bars, uint32_t base, volatile int32_t *failed, int32_t keys, int tile, int32_t last,
                                             int thread) {
    if (keys >= kTileKeys || (keys & 15) == 0) return true;
    using Smem = WideSmem<D>;
    const uint32_t stage = last % Smem::kStages;
    if (!wait_for_copy<Smem::kStages>(sh, bars, last, failed)) return false;
    const int32_t clear = ((keys + 15) & ~15) - keys;
    for (int32_t c = thread; c < clear * (D / 8); c += kHalfThreads) {
        const int32_t r = tile * kTileKeys + keys + c / (D / 8), chunk = c % (D / 8);
        store16(base + Smem::kRing + stage * Smem::kStageBytes + (chunk >> 3) * (kWideKeys * 128) + r * 128 + (chunk & 7) * 16, make_uint4(0, 0, 0, 0));
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    return true;
}

// One stream, by a whole CTA, with its tiles and WideShared at s_tiles.  All threads return together.
template <typename Q, int D>
__device__ __forceinline__ void wide_stream(const AttnArgs &a, const CUtensorMap &k_map, const CUtensorMap &v_map, uint8_t *s_tiles) {
    using Smem = WideSmem<D>;
    constexpr int kStages = Smem::kStages, kParts = D / 64;
    WideShared &sh = *reinterpret_cast<WideShared *>(s_tiles + Smem::kSmall);
    const uint32_t base = smem_at(s_tiles), at_bars = smem_at(sh.bars);
    const WideBars bars = {at_bars, at_bars + 8 * kStages, at_bars + 16 * kStages, at_bars + 16 * kStages + 32, at_bars + 16 * kStages + 64, at_bars + 16 * kStages + 80, at_bars + 16 * kStages + 96};
    static_assert(2 * kStages + 14 <= 40, "barriers");
    const int warp = threadIdx.x >> 5, lane = lane_id();
    bool bad = false;
    if ((int64_t)blockIdx.x * steps_per_stream<true>(a) >= __ldcg(a.start[1] + a.N + a.R)) return;       // nothing on this stream

    if (threadIdx.x == 0) {
        sh.failed = 0;
        sh.issued = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(bars.full + 8 * s, 1);
            bar_init(bars.empty + 8 * s, 2);             // both halves' products
        }
        for (int h = 0; h < 2; ++h) {
            for (int x = 0; x < 2; ++x) {
                bar_init(bars.scores + 16 * h + 8 * x, 1);
                bar_init(bars.weights + 16 * h + 8 * x, kHalfThreads);
            }
            bar_init(bars.queries + 8 * h, kHalfThreads);
            bar_init(bars.product + 8 * h, 1);
            bar_init(bars.output + 8 * h, 1);
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
    const uint32_t tmem = sh.tmem;                        // columns: S of the halves, 128 each, then O, D each
    volatile int32_t *failed = &sh.failed;

    // All warps go through the stream's pieces in batches: one warp lists a batch, the others work through it.  Returns how many there are.
    auto next_batch = [&]() {
        __syncthreads();
        return sh.failed ? 0 : sh.pieces;
    };
    if (warp >= kTmaWarp) {
        if (warp >= kListWarp) {
            Pieces<true> pieces(a, blockIdx.x, bad);
            int32_t n = 1;
            while (n > 0) {
                n = 0;
                Piece w;
                while (warp == kListWarp && n < kPieceBatch && pieces.next(a, w, bad)) {
                    if (lane == 0) {
                        WidePiece &p = sh.piece[n];
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
                if (warp == kListWarp && lane == 0) sh.pieces = n;
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
                if (lane_box < boxes && HORA_IN((key0 >> a.page_shift) + lane_box, p.prompt ? a.prefix_ld : a.suffix_ld)) id = __ldcg(p.pages + (key0 >> a.page_shift) + lane_box);
                if (id < 0 || id >= a.n_pages) { bad = true; id = 0; }
                if (pos >= kStages) ok = bar_wait(bars.empty + 8 * stage, (pos / kStages + 1) & 1, failed);
                ok = __all_sync(kFull, ok);
                if (!ok) return;
                if (lane == 0) {
                    bar_expect(bars.full + 8 * stage, boxes * page * D * 2);
                    __threadfence_block();
                    *const_cast<volatile int32_t *>(&sh.issued) = pos + 1;
                }
                __syncwarp();
                if (lane_box < boxes)
                    tma_box(base + Smem::kRing + stage * Smem::kStageBytes + lane_part * (kWideKeys * 128) + lane_box * page * 128, map, lane_part * 64,
                            (int32_t)(((int64_t)id * a.Hkv + p.h) << a.page_shift), bars.full + 8 * stage);
                ++pos;
            };
            while (const int32_t listed = next_batch()) {
                for (int32_t at = 0; at < listed && ok; ++at) {
                    const WidePiece &p = sh.piece[at];
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
        } else {
            // ---- products of one half
            const int half = warp - kMmaWarp;
            constexpr uint32_t kType = std::is_same<Q, __nv_bfloat16>::value ? 1u : 0u;
            constexpr uint32_t kIdescS = (1u << 4) | (kType << 7) | (kType << 10) | ((kTileKeys / 8) << 17) | ((kWideHalf / 16) << 24);
            constexpr uint32_t kIdescO = (1u << 4) | (kType << 7) | (kType << 10) | (1u << 16) | ((D / 8) << 17) | ((kWideHalf / 16) << 24);
            // the stages in the order of their first use
            uint32_t weights_phase = 0, queries_phase = 0;
            int32_t pos = 0;
            const uint32_t k0 = operand(base + Smem::kRing, 16), v0 = operand(base + Smem::kRing, kWideKeys * 128);
            const uint32_t q = operand(base + Smem::kQ + half * Smem::kQBytes, 16), t_s = tmem + half * 128, t_o = tmem + 256 + half * D;
            bool ok = true;
            auto next_stage = [&](bool mine, bool both) {           // the next one, once its copy has arrived if it is for this half
                const int32_t now = pos++;
                // where the half uses every stage it is never a whole ring behind
                if (mine) ok = ok && (both ? bar_wait(bars.full + 8 * (now % kStages), (now / kStages) & 1, failed) : wait_for_copy<kStages>(sh, bars, now, failed));
                return (uint32_t)(now % kStages);
            };
            auto release = [&](uint32_t used, bool both) {
                mma_commit(bars.empty + 8 * used);
                if (!both) mma_commit(bars.empty + 8 * used);
            };
            uint32_t k_used = 0, v_used = 0;
            while (const int32_t listed = next_batch()) {
                for (int32_t at = 0; at < listed && ok; ++at) {
                    const bool both = sh.piece[at].both;
                    const int32_t len = sh.piece[at].len, key0 = sh.piece[at].key0 + (both ? 0 : half * kWideKeys), stride = both ? kWideKeys : 2 * kWideKeys;
                    const int32_t n0 = sh.piece[at].count(0), n1 = sh.piece[at].count(1), tiles = sh.piece[at].tiles(half);
                    // scores of tile t, whose step's keys are in stage k_used
                    auto scores = [&](int32_t t) {
                        fence_after();
                        if (ok && elect_one()) {
                            const uint32_t k = k0 + k_used * (Smem::kStageBytes >> 4) + (t & 1) * ((kTileKeys * 128) >> 4), d = t_s + (t & 1) * kTileKeys;
#pragma unroll
                            for (int x = 0; x < D / 16; ++x) {
                                const uint32_t off = ((x >> 2) * (kWideKeys * 128) + (x & 3) * 32) >> 4;
                                mma_smem(d, q + off, k + off, kIdescS, x > 0);
                            }
                            mma_commit(bars.scores + 16 * half + 8 * (t & 1));
                            if ((t & 1) || t == tiles - 1) release(k_used, both);
                        }
                        __syncwarp();
                    };
                    auto product = [&](int32_t t) {
                        ok = ok && bar_wait(bars.weights + 16 * half + 8 * (t & 1), (weights_phase >> (t & 1)) & 1, failed);
                        weights_phase ^= 1u << (t & 1);
                        fence_after();
                        if (ok && elect_one()) {
                            const uint32_t v = v0 + v_used * (Smem::kStageBytes >> 4) + (t & 1) * ((kTileKeys * 128) >> 4), w = t_s + (t & 1) * kTileKeys;
                            const int32_t left = len - key0 - (t >> 1) * stride - (t & 1) * kTileKeys;
#pragma unroll
                            for (int g = 0; g < kTileKeys / 16; ++g)
                                if (g * 16 < left) mma_tmem(t_o, w + g * 8, v + g * (2048 >> 4), kIdescO, t > 0 || g > 0);
                            mma_commit(bars.product + 8 * half);
                            if ((t & 1) || t == tiles - 1) release(v_used, both);
                            if (t == tiles - 1) mma_commit(bars.output + 8 * half);
                        }
                        __syncwarp();
                    };
                    // stages come in the order in which the halves need them: for each of their steps, first the values of the step before
                    for (int32_t it = 0; it <= n0 && ok; ++it)
                        for (int turn = 0; turn < (both ? 1 : 2) && ok; ++turn) {
                            const bool mine = both || turn == half;
                            const int32_t nt = turn ? n1 : n0;
                            const bool values = it >= 1 && it - 1 < nt, keys = it < nt;
                            if (values) {
                                const uint32_t used = next_stage(mine, both);
                                if (mine) v_used = used;
                            }
                            if (mine && values) product(2 * it - 2);
                            if (keys) {
                                const uint32_t used = next_stage(mine, both);
                                if (mine) k_used = used;
                            }
                            if (!mine) continue;
                            if (keys) {
                                if (it == 0) {
                                    ok = ok && bar_wait(bars.queries + 8 * half, queries_phase, failed);
                                    queries_phase ^= 1;
                                }
                                scores(2 * it);
                            }
                            if (values && 2 * it - 1 < tiles) product(2 * it - 1);
                            if (keys && 2 * it + 1 < tiles) scores(2 * it + 1);
                        }
                }
                __syncthreads();
            }
            __syncthreads();
        }
    } else {
        // ---- softmax: thread `row` of a half has row `row` of its scores
        const int half = warp >> 2, row = threadIdx.x & (kWideHalf - 1);
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);           // this warp's 32 lanes of tensor memory
        const uint32_t t_s = lanes + half * 128, t_o = lanes + 256 + half * D;
        uint32_t scores_phase = 0, n_product = 0, n_output = 0;
        int32_t pos = 0;                                 // stages of all pieces before this one
        bool ok = true;
        while (const int32_t listed = next_batch()) {
            for (int32_t at = 0; at < listed && ok; ++at) {
                const WidePiece &p = sh.piece[at];
                const int32_t tiles = p.tiles(half);
                const int32_t x = (p.both ? half * kWideHalf : 0) + row;      // row of the item
                QueryRow qr = {-1, 0};
                if (x < p.rows) qr = query_row(a, p.first, p.seq_rows, p.len, p.prompt, p.h, p.row0 + x);
                const bool warp_has_rows = __any_sync(kFull, qr.out >= 0);
                float m = -INFINITY, l = 0.f;
                if (tiles > 0) {
                    // queries into shared memory, neighbouring lanes along a row; the products that read the last ones are done (their
                    // output was waited for)
                    if (warp_has_rows) {
                        const int64_t from = qr.out >= 0 ? qr.out / a.Hq * a.q_row_stride + qr.out % a.Hq * D : -1;
                        constexpr int kLanes = D / 8, kRows = kWarp / kLanes;             // lanes to a row, rows at a time
                        const int c = lane % kLanes;
#pragma unroll 8
                        for (int y = 0; y < kLanes; ++y) {
                            const int r = y * kRows + lane / kLanes;
                            const int64_t at_r = __shfl_sync(kFull, from, r);
                            const uint4 v = at_r >= 0 && HORA_IN(at_r + c * 8 + 7, (int64_t)a.R * a.T * a.q_row_stride) ? __ldcg(reinterpret_cast<const uint4 *>(static_cast<const Q *>(a.q) + at_r) + c) : make_uint4(0, 0, 0, 0);
                            const int qrow = (warp & 3) * kWarp + r;
                            store16(base + Smem::kQ + half * Smem::kQBytes + (c >> 3) * (kWideHalf * 128) + qrow * 128 + (((c & 7) ^ (qrow & 7)) << 4), v);
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    bar_arrive(bars.queries + 8 * half);
                    for (int32_t t = 0; t < tiles; ++t) {
                        const int32_t key0 = p.key(half, t >> 1) + (t & 1) * kTileKeys;
                        ok = ok && bar_wait(bars.scores + 16 * half + 8 * (t & 1), (scores_phase >> (t & 1)) & 1, failed);
                        scores_phase ^= 1u << (t & 1);
                        ok = __all_sync(kFull, ok);
                        if (!ok) break;
                        fence_after();
                        if (warp_has_rows) {
                            float s[2][32];
#pragma unroll
                            for (int b = 0; b < 2; ++b) tmem_load(t_s + (t & 1) * kTileKeys + b * 32, s[b]);
                            tmem_load_wait();
                            if (key0 + kTileKeys > qr.limit) {
#pragma unroll
                                for (int b = 0; b < 2; ++b)
#pragma unroll
                                    for (int e = 0; e < 32; ++e)
                                        if (key0 + b * 32 + e >= qr.limit) s[b][e] = -INFINITY;
                            }
                            float t4[4];
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                t4[b] = s[b >> 1][(b & 1) * 16];
#pragma unroll
                                for (int e = 1; e < 15; e += 2) t4[b] = fmaxf(t4[b], fmaxf(s[b >> 1][(b & 1) * 16 + e], s[b >> 1][(b & 1) * 16 + e + 1]));
                                t4[b] = fmaxf(t4[b], s[b >> 1][(b & 1) * 16 + 15]);
                            }
                            const float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])) * a.scale_log2;
                            if (t == 0) {
                                m = top;
                            } else if (__any_sync(kFull, top > m + 8.f)) {
                                // the last product has to be in before its output is scaled
                                ok = bar_wait(bars.product + 8 * half, (n_product + t - 1) & 1, failed);
                                ok = __all_sync(kFull, ok);
                                fence_after();
                                const float up = fmaxf(m, top), f = up == -INFINITY ? 1.f : exp2_fast(m - up);
                                l *= f;
                                m = up;
                                scale_output<D>(t_o, f);
                            }
                            // where no key has been seen the reference is -infinity and every weight has to come out as 0
                            const float z = m == -INFINITY ? 0.f : m;
                            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                uint32_t w[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    float2 y = make_float2(s[b >> 1][(b & 1) * 16 + 2 * e], s[b >> 1][(b & 1) * 16 + 2 * e + 1]);
                                    y = fma2(y, make_float2(a.scale_log2, a.scale_log2), make_float2(-z, -z));
                                    if (e % 4 == 3) y = exp2_by_products(y);
                                    else y = make_float2(exp2_fast(y.x), exp2_fast(y.y));
                                    sum = add2(sum, y);
                                    w[e] = pack2(y.x, y.y, Q());
                                }
                                tmem_store8(t_s + (t & 1) * kTileKeys + b * 8, w);
                            }
                            l += sum.x + sum.y;
                            tmem_store_wait();
                        }
                        if (t == tiles - 1) ok = clear_values<D>(sh, bars, base, failed, p.len - key0, t & 1, pos + 2 * p.n - 1, row) && ok;
                        fence_before();
                        bar_arrive(bars.weights + 16 * half + 8 * (t & 1));
                    }
                    n_product += tiles;
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
                if (qr.out >= 0 && HORA_IN(place, p.continued ? (int64_t)a.n_wide * kWideRows : 4 * rows_all)) *reinterpret_cast<float2 *>((p.continued ? a.cont_ml[1] : a.main_ml) + place * 2) = make_float2(m, l);
                if (tiles > 0) {
                    // through the warp's rows of the query tile, which nobody reads any more, so that neighbouring lanes store along a row
                    constexpr int kColumns = 32, kLanes = kColumns / 4, kRows = kWarp / kLanes;               // columns at a time
                    const uint32_t tile = base + Smem::kQ + half * Smem::kQBytes + (warp & 3) * (kWarp * 128);
                    float *__restrict__ po = p.continued ? a.cont_o[1] : a.main_o;
                    const int64_t from = qr.out >= 0 ? place * D : -1;
                    const int c = lane % kLanes;
#pragma unroll 1
                    for (int y = 0; y < D / kColumns; ++y) {
                        float o[kColumns];
                        tmem_load(t_o + y * kColumns, o);
                        tmem_load_wait();
                        __syncwarp();
#pragma unroll
                        for (int v = 0; v < kLanes; ++v)
                            store16(tile + lane * 128 + ((v ^ (lane & 7)) << 4),
                                    make_uint4(__float_as_uint(o[4 * v]), __float_as_uint(o[4 * v + 1]), __float_as_uint(o[4 * v + 2]), __float_as_uint(o[4 * v + 3])));
                        __syncwarp();
#pragma unroll
                        for (int v = 0; v < kLanes; ++v) {
                            const int r = v * kRows + lane / kLanes;
                            const int64_t to = __shfl_sync(kFull, from, r);
                            const uint4 got = load16(tile + r * 128 + ((c ^ (r & 7)) << 4));
                            if (to >= 0 && HORA_IN(to / D, p.continued ? (int64_t)a.n_wide * kWideRows : 4 * rows_all)) *reinterpret_cast<uint4 *>(po + to + y * kColumns + c * 4) = got;
                        }
                    }
                    __syncwarp();
                }
                fence_before();                          // the next item's products may overwrite O: its weights come after this
            }
            __syncthreads();
        }
        __syncthreads();
    }
    if (bad) raise_status(a.status, HORA_ERR_INVALID_VALUE);
    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && sh.failed) raise_status(a.status, HORA_ERR_INTERNAL);
    if (warp == 0) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

}  // namespace hora
