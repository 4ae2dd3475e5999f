// hora_group_attention: what its kernels share.
//
// The work is a list of N + R key sequences: the N prompts' (all queries of the group attend to them) and the R
// rollouts' own.  A sequence has `rows` query rows for each cache head: (rollout, slot t, head of the cache head's
// group), in that order.  A block of rows of a sequence and one cache head is an item; an item's keys come in steps.
// Sequences with few rows to a key are bound by the cache's bytes: their items are narrow (mma.sync, a warp to a stream);
// those with many have the products to do: theirs are wide (tcgen05, a CTA to a stream).  All steps of the narrow
// items, in order, form one line that is cut into equal pieces, one for each stream, and so do those of the wide items, so
// every stream has about the same to do whatever the lengths are.  A piece's part of an item is a partial
// result (m, l, o): m a reference score in units of log2, l = sum 2^(s - m), o = sum 2^(s - m) v.  Partials are joined at
// the end: m = max m_i, l = sum l_i 2^(m_i - m), o = sum o_i 2^(m_i - m), out = o / l.
//
// Where a partial goes: the part of an item that begins the item has a place of its own for each output row; a part
// that goes on with an item begun by an earlier stream is the first thing its stream does, so that one has a place for each stream.
#pragma once

#include "hora_checked.cuh"
#include "hora_rows16.cuh"

namespace hora {

// query rows of a narrow item: as many eights as a rollout's queries of one cache head need, while the registers last
constexpr int narrow_eights(int rows, int D) { return rows <= 8 ? 1 : rows <= 16 || D == 128 ? 2 : 3; }
// keys of its steps: 16 where that is 8 KiB, else 32 (twice the independent work between two looks at the maximum)
constexpr int narrow_keys(bool f8, int D) { return !f8 && D == 128 ? 16 : 32; }
constexpr int kNarrowPerSm = 12;                         // streams an SM: 168 registers a lane, 16 KiB of keys and values in flight each
constexpr int kAttnThreads = kNarrowPerSm * kWarp;
constexpr int kNarrowMinSteps = 4;                       // a stream shorter than this costs more to join than it saves

constexpr int kWideRows = 256;                           // query rows of a wide item, in two halves
constexpr int kWideHalf = kWideRows / 2;
constexpr int kWideKeys = 128;
constexpr int kWideFrom = 33, kWideLong = 1024;          // rows from which, keys from which a sequence's items can be wide

// Parts that a row's result is joined from, other than the continued ones.
enum { kPromptPart = 0, kOwnPart = 1, kSecondHalf = 2 }; // kSecondHalf: added for the second half of the keys (wide items of one half)

struct AttnArgs {
    const void *q;
    const int64_t *group_offsets;
    const int32_t *q_len, *prefix_pages, *prefix_len, *suffix_pages, *suffix_len;
    const void *k_cache, *v_cache;
    const uint8_t *k_exp, *v_exp;
    void *out;
    float *lse;
    int32_t *status;
    int64_t q_row_stride, out_row_stride, n_pages;
    int32_t N, R, T, Hq, Hkv, g, page_shift, prefix_ld, suffix_ld;
    int32_t n_sm, n_narrow, n_wide;                      // CTAs, streams of each line; n_wide 0: every sequence is narrow
    int32_t narrow_keys, narrow_rows;                    // keys of a narrow step, rows of a narrow item
    float scale_log2;                                    // sm_scale * log2(e)
    // workspace
    int64_t *start[2];                                   // [N + R + 3] first step of each sequence on the narrow, the wide line; all; a stream's; [1]: has_wide
    int32_t *group_of;                                   // [R] group of each rollout, -1: none
    float *main_o, *main_ml;                             // [2 or 4][R * T * Hq][D], [..][2], by part
    float *cont_o[2], *cont_ml[2];                       // [streams][rows of an item][D], [..][2]
};

// A sequence: its query rows per cache head, its keys, and how it is cut.
struct Sequence {
    int32_t first, rollouts;                             // rollouts that attend to it
    int32_t rows, len, steps, tiles, tile_rows;
    bool wide;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ int32_t clamp_i64(int64_t v, int32_t lo, int32_t hi) { return v < lo ? lo : (v > hi ? hi : (int32_t)v); }

__device__ __forceinline__ int32_t checked_len(int32_t len, int32_t ld, int32_t page_shift, bool &bad) {
    const int64_t room = (int64_t)ld << page_shift;
    if (len < 0 || len > room) bad = true;
    return len < 0 ? 0 : (len > room ? (int32_t)room : len);
}

__device__ __forceinline__ int32_t query_count(const AttnArgs &a, int32_t r) {
    const int32_t n = a.q_len ? __ldcg(a.q_len + r) : a.T;
    return n < 0 ? 0 : (n > a.T ? a.T : n);
}

// Whether a sequence's items can be wide.  Many rows: a narrow item would read the keys again for every eight or sixteen of them.  Fewer rows
// over a long list: the same, and the CTA's 128 rows may be mostly idle, since the bytes are what takes the time (103485 keys,
// 32 rows of 4 heads each: 318 us as narrow items, 122 as wide ones).  Short lists of few rows are narrow: a piece of a wide item costs
// some microseconds to begin and to end (256 rollouts of 20 rows over up to 1021 keys: 122 us, 172 as wide items).
//   From kWideFrom rows on the length does not enter, which costs short lists: 600 rollouts, 4 cache heads, us as wide / as narrow items
//     D = 64:  40 rows, 128 keys 95 / 89, 1024 keys 361 / 242;  128 rows, 128 keys 221 / 221, 1024 keys 426 / 652
//     D = 128: 40 rows, 128 keys 189 / 137, 1024 keys 424 / 503;  128 rows, 64 keys 266 / 245, 1024 keys 518 / 1303
__device__ __forceinline__ bool can_be_wide(const AttnArgs &a, const Sequence &s) {
    return a.n_wide > 0 && (s.rows >= kWideFrom || (s.rows > a.narrow_rows && s.len >= kWideLong));
}

// `wide`: whether sequences that can be are wide in this call.
__device__ __forceinline__ Sequence sequence(const AttnArgs &a, int32_t i, bool wide, bool &bad) {
    Sequence s = {};
    if (!HORA_IN(i, a.N + a.R)) return s;
    if (i < a.N) {
        const int64_t lo = __ldcg(a.group_offsets + i), hi = __ldcg(a.group_offsets + i + 1);
        if (lo < 0 || hi < lo || hi > a.R || (i == 0 && lo != 0)) bad = true;
        s.first = clamp_i64(lo, 0, a.R);
        s.rollouts = clamp_i64(hi, s.first, a.R) - s.first;
        s.len = checked_len(__ldcg(a.prefix_len + i), a.prefix_ld, a.page_shift, bad);
    } else {
        s.first = i - a.N;
        const int32_t n = a.q_len ? __ldcg(a.q_len + s.first) : a.T;
        if (n < 0 || n > a.T) bad = true;
        s.rollouts = s.first < __ldcg(a.group_offsets + a.N) ? 1 : 0;
        s.len = checked_len(__ldcg(a.suffix_len + s.first), a.suffix_ld, a.page_shift, bad);
    }
    s.rows = s.rollouts * a.T * a.g;
    s.wide = wide && can_be_wide(a, s);
    if (s.wide) {                                        // blocks of about the same size, so that their steps take the same time
        s.tiles = (s.rows + kWideRows - 1) / kWideRows;
        s.tile_rows = (s.rows + s.tiles - 1) / s.tiles;
        s.steps = (s.len + kWideKeys - 1) / kWideKeys;
    } else {
        s.tiles = (s.rows + a.narrow_rows - 1) / a.narrow_rows;
        s.tile_rows = a.narrow_rows;
        s.steps = (s.len + a.narrow_keys - 1) / a.narrow_keys;
    }
    return s;
}

__device__ __forceinline__ int64_t total_steps(const AttnArgs &a, const Sequence &s) { return (int64_t)s.steps * s.tiles * a.Hkv; }

// Steps of a line that go to one stream; the plan leaves it behind the line's starts.
template <bool WIDE>
__device__ __forceinline__ int64_t steps_per_stream(const AttnArgs &a) { return __ldcg(a.start[WIDE] + a.N + a.R + 1); }
// Whether the call has wide items: the plan leaves that there too.
__device__ __forceinline__ bool has_wide(const AttnArgs &a) { return __ldcg(a.start[1] + a.N + a.R + 2) != 0; }

// A stream's part of one item.
struct Piece {
    int32_t h, row0, rows, step0, step1;
    bool prompt;
    const int32_t *pages;
};

// Walks a stream's pieces in order; `s` is the sequence of the last one.  All lanes of a warp together.
template <bool WIDE>
struct Pieces {
    int64_t u, u_end, s_start;
    int32_t i;
    bool wide;
    Sequence s;

    __device__ __forceinline__ Pieces(const AttnArgs &a, int32_t stream, bool &bad) {
        const int64_t *start = a.start[WIDE];
        const int32_t n_seq = a.N + a.R;
        const int64_t per = steps_per_stream<WIDE>(a);
        u = (int64_t)stream * per;
        u_end = min(__ldcg(start + n_seq), u + per);
        i = 0;
        if (u >= u_end) return;
        for (int32_t hi = n_seq; hi - i > 1;) {          // start[i] <= u < start[hi], 32 probes at a time
            const int32_t gap = (hi - i + kWarp - 1) / kWarp;
            const int32_t probe = min(hi, i + lane_id() * gap);
            const unsigned at_or_before = __ballot_sync(kFull, probe < hi && __ldcg(start + probe) <= u);
            const int32_t top = 31 - __clz(at_or_before); // lane 0 always is
            hi = min(hi, i + (top + 1) * gap);
            i += top * gap;
        }
        wide = has_wide(a);
        s = sequence(a, i, wide, bad);
        s_start = __ldcg(start + i);
    }

    __device__ __forceinline__ bool next(const AttnArgs &a, Piece &p, bool &bad) {
        if (u >= u_end) return false;
        while (s.wide != WIDE || u >= s_start + total_steps(a, s)) {        // on to the next sequence with steps on this line
            if (i + 1 >= a.N + a.R) {                    // lengths that have changed since the plan: nothing beyond the last sequence is read
                (void)HORA_IN(i + 1, a.N + a.R);
                bad = true;
                return false;
            }
            if (s.wide == WIDE) s_start += total_steps(a, s);
            s = sequence(a, ++i, wide, bad);
        }
        const int64_t item = (u - s_start) / s.steps;
        p.step0 = (int32_t)((u - s_start) - item * s.steps);
        p.step1 = (int32_t)min((int64_t)s.steps, p.step0 + (u_end - u));
        p.h = (int32_t)(item / s.tiles);
        p.row0 = (int32_t)(item % s.tiles) * s.tile_rows;
        p.rows = min(s.tile_rows, s.rows - p.row0);
        p.prompt = i < a.N;
        p.pages = p.prompt ? a.prefix_pages + (int64_t)i * a.prefix_ld : a.suffix_pages + (int64_t)(i - a.N) * a.suffix_ld;
        u += p.step1 - p.step0;
        return true;
    }
};

// A row of an item: which query it is and how many of the sequence's keys it sees.
struct QueryRow {
    int64_t out;                                         // (rollout * T + t) * Hq + head, -1: no such row
    int32_t limit;
};

// Row x of a sequence and cache head h, for a sequence of `rows` rows and `len` keys whose first rollout is `first`.
__device__ __forceinline__ QueryRow query_row(const AttnArgs &a, int32_t first, int32_t rows, int32_t len, bool prompt, int32_t h, int32_t x) {
    QueryRow q = {-1, 0};
    if (x >= rows) return q;
    const int32_t per = a.T * a.g;
    const int32_t r = first + x / per, rem = x % per, t = rem / a.g;
    const int32_t n = query_count(a, r);
    q.out = ((int64_t)r * a.T + t) * a.Hq + h * a.g + rem % a.g;
    if (t >= n) return q;
    q.limit = prompt ? len : max(0, min(len, len - n + t + 1));
    return q;
}

hora_status_t launch_attention_main(const AttnArgs &a, int32_t q_dtype, int32_t cache_dtype, int32_t D, cudaStream_t stream);

}  // namespace hora
