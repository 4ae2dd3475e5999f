// hora_group_attention: what its kernels share.
//
// The work is a list of N + R key sequences: the N prompts' (all queries of the group attend to them) and the R
// rollouts' own.  A sequence has `rows` query rows for each cache head: (rollout, slot t, head of the cache head's
// group), in that order.  A row tile of a sequence and one cache head is an item; an item's keys come in steps.  All steps
// of all items, in order, form one line that is cut into equal pieces, one for each stream (a warp that runs by itself), so
// every stream reads about the same number of bytes whatever the lengths are.  A piece's part of an item is a partial
// result (m, l, o): m the largest score in units of log2, l = sum 2^(s - m), o = sum 2^(s - m) v.  Partials are joined at
// the end: m = max m_i, l = sum l_i 2^(m_i - m), o = sum o_i 2^(m_i - m), out = o / l.
//
// Where a partial goes: the part of an item that begins the item has a place of its own for each output row; a part
// that goes on with an item begun by an earlier stream is the first thing its stream does, so that one has a place for each stream.
#pragma once

#include "hora_rows16.cuh"

namespace hora {

constexpr int kTileRows = 16;                            // query rows of an item
constexpr int kStepKeys = 16;                            // keys of a step
constexpr int kStreamsPerSm = 12;                       // 168 registers a lane, 16 KiB of keys and values in flight each
constexpr int kMinSteps = 4;                             // a stream shorter than this costs more to join than it saves

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
    int32_t n_streams;
    float scale_log2;                                    // sm_scale * log2(e)
    // workspace
    int64_t *start;                                      // [N + R + 1] first step of each sequence on the line
    int32_t *group_of;                                   // [R] group of each rollout, -1: none
    float *main_o, *main_ml;                             // [2][R * T * Hq][D], [..][2]: prompt part, own part
    float *cont_o, *cont_ml;                             // [n_streams][kTileRows][D], [..][2]
};

// A sequence: its query rows per cache head, its keys, and how it is cut.
struct Sequence {
    int32_t first, rollouts;                             // rollouts that attend to it
    int32_t rows, len, steps, tiles;
};

__device__ __forceinline__ int32_t clamp_i64(int64_t v, int32_t lo, int32_t hi) { return v < lo ? lo : (v > hi ? hi : (int32_t)v); }

__device__ __forceinline__ int32_t checked_len(int32_t len, int32_t ld, int32_t page_shift, bool &bad) {
    const int64_t room = (int64_t)ld << page_shift;
    if (len < 0 || len > room) bad = true;
    return len < 0 ? 0 : (len > room ? (int32_t)room : len);
}

__device__ __forceinline__ int32_t query_count(const AttnArgs &a, int32_t r) {
    const int32_t n = a.q_len ? __ldg(a.q_len + r) : a.T;
    return n < 0 ? 0 : (n > a.T ? a.T : n);
}

__device__ __forceinline__ Sequence sequence(const AttnArgs &a, int32_t i, bool &bad) {
    Sequence s;
    if (i < a.N) {
        const int64_t lo = __ldg(a.group_offsets + i), hi = __ldg(a.group_offsets + i + 1);
        if (lo < 0 || hi < lo || hi > a.R || (i == 0 && lo != 0)) bad = true;
        s.first = clamp_i64(lo, 0, a.R);
        s.rollouts = clamp_i64(hi, s.first, a.R) - s.first;
        s.len = checked_len(__ldg(a.prefix_len + i), a.prefix_ld, a.page_shift, bad);
    } else {
        s.first = i - a.N;
        const int32_t n = a.q_len ? __ldg(a.q_len + s.first) : a.T;
        if (n < 0 || n > a.T) bad = true;
        s.rollouts = s.first < __ldg(a.group_offsets + a.N) ? 1 : 0;
        s.len = checked_len(__ldg(a.suffix_len + s.first), a.suffix_ld, a.page_shift, bad);
    }
    s.rows = s.rollouts * a.T * a.g;
    s.steps = (s.len + kStepKeys - 1) / kStepKeys;
    s.tiles = (s.rows + kTileRows - 1) / kTileRows;
    return s;
}

// Steps of the line that go to one stream.
__device__ __forceinline__ int64_t steps_per_stream(const AttnArgs &a) {
    const int64_t total = __ldg(a.start + a.N + a.R);
    return max((int64_t)kMinSteps, (total + a.n_streams - 1) / a.n_streams);
}

// A row of an item: which query it is and how many of the sequence's keys it sees.
struct QueryRow {
    int64_t out;                                         // (rollout * T + t) * Hq + head, -1: no such row
    int32_t limit;
};

__device__ __forceinline__ QueryRow query_row(const AttnArgs &a, const Sequence &s, bool prompt, int32_t h, int32_t x) {
    QueryRow q = {-1, 0};
    if (x >= s.rows) return q;
    const int32_t per = a.T * a.g;
    const int32_t r = s.first + x / per, rem = x % per, t = rem / a.g;
    const int32_t n = query_count(a, r);
    q.out = ((int64_t)r * a.T + t) * a.Hq + h * a.g + rem % a.g;
    if (t >= n) return q;
    q.limit = prompt ? s.len : max(0, min(s.len, s.len - n + t + 1));
    return q;
}

hora_status_t launch_attention_plan(const AttnArgs &a, cudaStream_t stream);
hora_status_t launch_attention_steps(const AttnArgs &a, int32_t q_dtype, int32_t cache_dtype, int32_t D, cudaStream_t stream);
hora_status_t launch_attention_join(const AttnArgs &a, int32_t q_dtype, int32_t D, cudaStream_t stream);

}  // namespace hora
