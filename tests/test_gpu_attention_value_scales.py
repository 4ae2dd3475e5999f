"""hora_group_attention over an e4m3 cache whose value rows differ widely in scale, against the definition in 64 bits.

Tolerance.  A weight enters the product in fp16, times its row's scale, relative to a reference r that is at most the largest such product W
among the keys that the query sees (rows of zeros aside): off by 2^-11 of itself, or by 2^-25 r below fp16's normal range.  The latter
makes at most n 2^-25 W 448 of the sum over n keys.  The row with the product W has a code of 224 or more, so that in its dimension sum w |v| is at
least 224 W: n 2^-24 of the largest sum w |v| among the dimensions.  Scores are fp32 sums of D products, off by D 2^-23 sum |q k| scale, twice that
in an exponent's difference, and scale exponents up to 2^7 are added to them: 2^-16 with the exponential itself.  The output is rounded once.  There is no
term that grows with the values of keys that hardly count."""
from __future__ import annotations

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import decode as orc  # noqa: E402

DEV = "cuda"
F8 = torch.float8_e4m3fn
OUT = {torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}     # relative; absolute, below the normal range


@pytest.fixture(params=["normal", "checked"])
def hora(request):
    from paper_2605_07114_b200 import build as b, hora
    if request.param == "checked":
        hora.use_library(b.build(checked=True))
        assert hora.hora_checked_violation() == 0
    yield hora
    left = hora.hora_checked_violation() if request.param == "checked" else 0
    hora.use_library(None)
    assert left == 0, f"index check failed: file {left >> 20}, line {left & 0xFFFFF}"


def run(hora, sizes, plen, slen, T, q_len, Hq, Hkv, D, dtype, keys, values, q, page=16):
    """keys, values: functions of (sequence, n) giving [n, Hkv, D] fp32 rows, sequences in the order prompts, rollouts."""
    N, R = len(sizes), sum(sizes)
    lens = list(plen) + list(slen)
    need = [max(1, -(-n // page)) for n in lens]
    first = np.concatenate([[0], np.cumsum(need)])
    cache = hora.PagedCache.empty(int(first[-1]), page, Hkv, D, F8)
    pools = [np.zeros((int(first[-1]), Hkv, page, D)) for _ in range(2)]
    table = np.zeros((N + R, max(need)), np.int32)
    for i, n in enumerate(lens):
        table[i, :need[i]] = first[i] + np.arange(need[i])
        if n == 0:
            continue
        rows = [np.asarray(f(i, n), np.float32) for f in (keys, values)]
        cache.write(*(torch.from_numpy(x).to(DEV) for x in rows), torch.arange(n, device=DEV) + int(first[i]) * page)
        for pool, x in zip(pools, rows):
            for j in range(n):
                for h in range(Hkv):
                    codes, e = orc.quantise_row(x[j, h])
                    pool[first[i] + j // page, h, j % page] = orc.VALUES[codes] * 2.0 ** (e - 127)
    d = lambda a, t=torch.int32: torch.as_tensor(np.ascontiguousarray(a), dtype=t, device=DEV)  # noqa: E731
    off = np.concatenate([[0], np.cumsum(sizes)])
    qd = torch.from_numpy(q).to(dtype).to(DEV)
    op = hora.GroupAttention(cache, Hq, T, dtype, group_offsets=d(off, torch.int64), prefix_pages=d(table[:N]), prefix_len=d(plen), suffix_pages=d(table[N:]),
                             suffix_len=d(slen), q_len=d(q_len))
    out, lse = op.run(qd)
    torch.cuda.synchronize()
    want, wlse, bound, reach = orc.group_attention(qd.double().cpu().numpy(), off, q_len, D ** -0.5, *pools, table[:N], plen, table[N:], slen)
    ds = D * 2.0 ** -23 * reach
    n = max(plen) + max(slen)
    u, small = OUT[dtype]
    tol = bound * (2.0 ** -11 + 2 * ds[..., None] + 2.0 ** -16) + n * 2.0 ** -24 * bound.max(-1, keepdims=True) + u * np.abs(want) + small
    got = out.double().cpu().numpy()
    bad = np.argwhere(~(np.abs(got - want) <= tol))
    assert not len(bad), (len(bad), bad[0], got[tuple(bad[0])], want[tuple(bad[0])], tol[tuple(bad[0])])
    gl, seen = lse.double().cpu().numpy(), np.isfinite(wlse)
    assert (gl[~seen] == -math.inf).all() and (np.abs(gl[seen] - wlse[seen]) <= ds[seen] + 2.0 ** -18 * (1 + np.abs(wlse[seen]))).all()
    return got


SHAPES = [(8, 2, 64, 1), (8, 1, 128, 1), (12, 1, 64, 2), (16, 1, 128, 3)]               # Hq, Hkv, D, T: narrow items of 8, 16 and 24 rows


@pytest.mark.parametrize("Hq,Hkv,D,T", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("what", ["spread", "zeros", "mostly zeros", "all zeros", "tiny", "huge", "growing"])
def test_value_rows_of_very_different_scales(hora, what, dtype, Hq, Hkv, D, T):
    rng = np.random.default_rng(D + T)
    if dtype == torch.float16 and what in ("tiny", "huge"):
        pytest.skip("beyond the output type")

    def values(i, n):
        x = rng.standard_normal((n, Hkv, D))
        if what == "spread":
            return x * np.exp2(rng.integers(-24, 1, (n, Hkv, 1)))
        if what == "zeros":                                 # a null key now and then among small values
            return np.where(np.arange(n)[:, None, None] % 37 == 3, 0.0, 1e-4 * x)
        if what == "mostly zeros":
            return np.where(np.arange(n)[:, None, None] % 5 != 3, 0.0, 1e-4 * x) * np.where(rng.random((n, Hkv, D)) < 0.5, -1.0, 1.0)
        if what == "all zeros":
            return 0.0 * x
        if what == "tiny":
            return x * np.exp2(rng.integers(-110, -90, (n, Hkv, 1)))
        if what == "huge":
            return x * np.exp2(rng.integers(70, 110, (n, Hkv, 1)))
        return x * np.exp2(np.minimum(np.arange(n), 300) / 12 - 24)[:, None, None]

    q = rng.standard_normal((5, T, Hq, D))
    got = run(hora, [3, 2], [210, 33], [1, 40, 0, 70, 16], T, [min(T, x) for x in (1, 3, 0, 2, 3)], Hq, Hkv, D, dtype, lambda i, n: rng.standard_normal((n, Hkv, D)), values, q)
    assert what != "all zeros" or (got == 0).all()


@pytest.mark.parametrize("Hq,Hkv,D,T", SHAPES)
@pytest.mark.parametrize("gap", [12, 20, 30, 60])
def test_a_large_value_row_of_a_key_that_hardly_counts(hora, gap, Hq, Hkv, D, T):
    """One key opposite to the queries, about 2^-57 of a weight, with values 2^gap times the others': at the beginning, inside, at the end."""
    rng = np.random.default_rng(gap)
    base = rng.standard_normal(D)

    def keys(i, n):
        k = 0.1 * rng.standard_normal((n, Hkv, D))
        k[[0, n // 2, n - 1]] = -base * 57 * math.log(2) * math.sqrt(D) / (base @ base)
        return k

    def values(i, n):
        v = rng.standard_normal((n, Hkv, D))
        v[[0, n // 2, n - 1]] *= 2.0 ** gap
        return v

    q = np.broadcast_to(base, (4, T, Hq, D)) + 0.1 * rng.standard_normal((4, T, Hq, D))
    run(hora, [3, 1], [150, 70], [35, 17, 64, 3], T, [min(T, 3)] * 4, Hq, Hkv, D, torch.bfloat16, keys, values, q)


@pytest.mark.parametrize("Hq,Hkv,D,T", SHAPES[2:])
def test_large_value_rows_of_drafts_that_a_query_does_not_see(hora, Hq, Hkv, D, T):
    rng = np.random.default_rng(1)
    slen = [T, 20, 33]

    def values(i, n):
        v = rng.standard_normal((n, Hkv, D))
        if i >= 1:
            v[n - 1] *= 2.0 ** 40                           # the last draft of each rollout, seen by the last query alone
        return v

    run(hora, [3], [40], slen, T, [T] * 3, Hq, Hkv, D, torch.bfloat16, lambda i, n: rng.standard_normal((n, Hkv, D)), values, rng.standard_normal((3, T, Hq, D)))
