"""The decode-step operators from their definitions, in 64 bits: rows of a quantised cache, attention of rollout groups,
verification of drafted tokens.  numpy and Python integers only; one row, one query, one rollout at a time."""
from __future__ import annotations

import math

import numpy as np

GRID_BITS = 38


def e4m3_value(code: int) -> float:
    """Value of an e4m3 code: sign, 4 exponent bits (bias 7), 3 of significand; S.1111.111 is NaN, there is no infinity."""
    sign = -1.0 if code & 0x80 else 1.0
    e, m = (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return math.nan
    return sign * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))


VALUES = np.array([e4m3_value(c) for c in range(256)])
_POSITIVE = VALUES[:127]                                  # codes 0 .. 126 in increasing order of value


def quantise_row(x: np.ndarray):
    """(codes, biased exponent) of one row."""
    x = np.asarray(x, np.float64)
    finite = np.abs(x[np.isfinite(x)])
    top = finite.max() if finite.size else 0.0
    e = 0
    if top > 0:
        e = -126
        while top / 2.0 ** e > 448.0:
            e += 1
    codes = np.zeros(x.shape, np.uint8)
    for i, v in enumerate(x):
        if math.isnan(v):
            codes[i] = 127
            continue
        a = min(abs(v) / 2.0 ** e, 448.0)
        hi = int(np.searchsorted(_POSITIVE, a))           # first code with a value >= a
        if hi > 0 and _POSITIVE[min(hi, 126)] != a:
            lo, hi = hi - 1, min(hi, 126)
            dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
            hi = lo if dl < dh or (dl == dh and lo % 2 == 0) else hi
        codes[i] = hi | (128 if math.copysign(1.0, v) < 0 else 0)
    return codes, e + 127


def attention_query(q, k, v, scale):
    """One query over the keys it sees.  q [D], k, v [n, D] in 64 bits.  Returns (out, lse, bound): bound[d] = sum of the
    weights times |v_d|, what a relative error of the weights can make of the output; and the largest sum |q_i k_i| scale."""
    D = q.shape[0]
    if k.shape[0] == 0:
        return np.zeros(D), -math.inf, np.zeros(D), 0.0
    s = scale * (k @ q)
    m = s.max()
    w = np.exp(s - m)
    l = w.sum()
    return (w @ v) / l, m + math.log(l), (w @ np.abs(v)) / l, float(scale * (np.abs(k) @ np.abs(q)).max())


def group_attention(q, group_offsets, q_len, scale, k, v, prefix_pages, prefix_len, suffix_pages, suffix_len):
    """q [R, T, Hq, D], pools k, v [n_pages, H, page, D] as values, all in 64 bits.  Returns out, lse, bound, reach."""
    R, T, Hq, D = q.shape
    H, page = k.shape[1], k.shape[2]
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.full((R, T, Hq), -math.inf), np.zeros((R, T, Hq))

    def rows(pool, pages, h, n):
        got = [pool[pages[j // page], h, j % page] for j in range(n)]
        return np.array(got).reshape(n, D)

    for i in range(len(prefix_len)):
        for r in range(int(group_offsets[i]), int(group_offsets[i + 1])):
            n = int(q_len[r])
            for h in range(H):
                kp, vp = rows(k, prefix_pages[i], h, int(prefix_len[i])), rows(v, prefix_pages[i], h, int(prefix_len[i]))
                ks, vs = rows(k, suffix_pages[r], h, int(suffix_len[r])), rows(v, suffix_pages[r], h, int(suffix_len[r]))
                for t in range(n):
                    seen = max(0, int(suffix_len[r]) - n + t + 1)
                    kk, vv = np.concatenate([kp, ks[:seen]]), np.concatenate([vp, vs[:seen]])
                    for x in range(h * (Hq // H), (h + 1) * (Hq // H)):
                        out[r, t, x], lse[r, t, x], bound[r, t, x], reach[r, t, x] = attention_query(q[r, t, x], kk, vv, scale)
    return out, lse, bound, reach


def grid(p: float) -> int:
    """p, clamped to [0, 1], in units of 2^-38, rounded down; NaN counts as 0."""
    return 0 if not p > 0 else int(math.floor(min(p, 1.0) * 2 ** GRID_BITS))


def verify(target, draft, tokens, length, u_accept, u_sample):
    """One rollout.  target [K+1, V], draft [K, V] or None, tokens [K], u_accept [K].  Returns (n_accepted, tokens out)."""
    from fractions import Fraction
    K, V = len(tokens), len(target[0])
    n = 0
    while n < length:
        x = int(tokens[n])
        if not 0 <= x < V:
            break
        p, q = float(target[n][x]), 1.0 if draft is None else float(draft[n][x])
        if math.isnan(p) or math.isnan(q) or not Fraction(float(u_accept[n])) * Fraction(q) < Fraction(p):
            break
        n += 1
    plus = [grid(float(p)) for p in target[n]]
    w = plus
    if n < length:
        minus = [0] * V
        if draft is not None:
            minus = [grid(float(q)) for q in draft[n]]
        elif 0 <= int(tokens[n]) < V:
            minus[int(tokens[n])] = 1 << GRID_BITS
        w = [max(a - b, 0) for a, b in zip(plus, minus)]
        if not any(w):
            w = plus
    out = [int(x) for x in tokens[:n]] + [-1] * (K + 1 - n)
    total = sum(w)
    if total:
        limit = (total * int(math.floor(float(u_sample) * 2 ** 24))) >> 24
        run = 0
        for v, x in enumerate(w):
            run += x
            if run > limit:
                out[n] = v
                break
    return n, out
