"""hora_group_attention against the definition in 64 bits.

Tolerance.  The weights enter the product rounded to 16 bits: relative error u = 2^-8 (bf16) or 2^-11 (fp16, also used for
an e4m3 cache), below fp16's normal range 2^-25 absolute; the output is rounded once more.  With A = sum w |v| / sum w the
output is off by at most u A + u' |out| + 2^-25 n max|v|.  Scores are fp32 sums of D exact products: off by at most
D 2^-23 sum |q k| scale, twice that in the exponent's difference; the exponential itself and the sums add less than 2^-18 relative."""
from __future__ import annotations

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import decode as orc  # noqa: E402

DEV = "cuda"
F8 = torch.float8_e4m3fn
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _hora():
    from paper_2605_07114_b200 import hora
    return hora


@pytest.fixture(params=["normal", "checked"])
def build(request):
    """The tests run through the normal build and through the checked one, whose index checks have to stay silent and which
    gives every item with enough rows to the wide kernel (the normal build leaves problems as small as these to the narrow one)."""
    from paper_2605_07114_b200 import build as b
    hora = _hora()
    if request.param == "checked":
        hora.use_library(b.build(checked=True))
        assert hora.hora_checked_violation() == 0
    yield request.param
    left = hora.hora_checked_violation() if request.param == "checked" else 0
    hora.use_library(None)
    assert left == 0, f"index check failed: file {left >> 20}, line {left & 0xFFFFF}"


def make(sizes, prefix, suffix, T, Hq, Hkv, D, dtype, cache, page, seed, q_len=None, extra_rollouts=0, stride_extra=0, garbage=True, q_scale=2.0):
    """Everything a call takes, on the device, and the same on the host in 64 bits.  Unused slots hold NaN."""
    rng = np.random.default_rng(seed)
    N, R = len(sizes), int(sum(sizes)) + extra_rollouts
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    plen = np.asarray(prefix, np.int32)
    slen = np.asarray(suffix, np.int32)
    assert len(plen) == N and len(slen) == R
    ql = np.full(R, T, np.int32) if q_len is None else np.asarray(q_len, np.int32)
    lens = np.concatenate([plen, slen])
    need = -(-lens // page)
    n_pages = int(need.sum()) + 2
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((N + R, max(1, int(need.max())) + 1), -7, np.int32)     # entries beyond a length are never looked at
    used = np.zeros((n_pages, page), bool)
    at = 0
    for i, (w, n) in enumerate(zip(need, lens)):
        table[i, :w] = order[at:at + w]
        for j in range(w):
            used[order[at + j], :min(page, n - j * page)] = True
        at += w
    t = {}
    pools = []
    for name in "kv":
        x = rng.standard_normal((n_pages, Hkv, page, D))
        if cache == F8:
            codes = rng.integers(0, 256, (n_pages, Hkv, page, D)).astype(np.uint8)
            codes[(codes & 0x7F) == 0x7F] = 0x55
            exps = rng.integers(118, 121, (n_pages, Hkv, page)).astype(np.uint8)
            values = orc.VALUES[codes] * np.exp2(exps.astype(np.float64) - 127)[..., None]
            if garbage:
                codes.transpose(0, 2, 1, 3)[~used] = 0x7F
                exps.transpose(0, 2, 1)[~used] = 255
            t[name] = torch.from_numpy(codes).to(DEV).view(F8)
            t[name + "_exp"] = torch.from_numpy(exps).to(DEV)
        else:
            y = torch.from_numpy(x).to(dtype)
            values = y.double().numpy()
            if garbage:
                y.transpose(1, 2)[torch.from_numpy(~used)] = math.nan
            t[name], t[name + "_exp"] = y.to(DEV), None
        pools.append(values)
    q = torch.zeros(R, T, Hq * D + stride_extra, dtype=dtype)
    q[..., :Hq * D] = (q_scale * torch.from_numpy(rng.standard_normal((R, T, Hq * D)))).to(dtype)
    qd = q.to(DEV)[..., :Hq * D].unflatten(2, (Hq, D))
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    t.update(q=qd, off=d(off), q_len=None if q_len is None else d(ql), pp=d(table[:N]), pl=d(plen), sp=d(table[N:]), sl=d(slen))
    host = dict(q=q[..., :Hq * D].double().numpy().reshape(R, T, Hq, D), off=off, ql=ql, k=pools[0], v=pools[1], pp=table[:N], pl=plen, sp=table[N:], sl=slen)
    return t, host


def call(t, scale, out=None, status=None):
    hora = _hora()
    R, T, Hq, D = t["q"].shape
    N, Hkv = t["pl"].shape[0], t["k"].shape[1]
    ws = torch.full((hora.hora_group_attention_workspace_bytes(N, R, T, Hq, Hkv, D),), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full((R, T, Hq, D), 9.0, dtype=t["q"].dtype, device=DEV) if out is None else out
    lse = torch.full((R, T, Hq), 9.0, device=DEV)
    hora.hora_group_attention(t["q"], t["off"], t["q_len"], scale, t["k"], t["v"], t["k_exp"], t["v_exp"], t["pp"], t["pl"], t["sp"], t["sl"],
                              out, lse, ws, status)
    torch.cuda.synchronize()
    return out, lse


def check(t, h, scale, out, lse):
    want, wlse, bound, reach = orc.group_attention(h["q"], h["off"], h["ql"], scale, h["k"], h["v"], h["pp"], h["pl"], h["sp"], h["sl"])
    dtype, D = t["q"].dtype, h["q"].shape[-1]
    u_out = UNIT[dtype]
    u_w = 2.0 ** -11 if t["k"].dtype == F8 else u_out
    ds = D * 2.0 ** -23 * reach
    n = int(h["pl"].max(initial=0)) + int(h["sl"].max(initial=0))
    small = 0.0 if u_w == 2.0 ** -8 else 2.0 ** -25 * n * np.abs(np.nan_to_num(h["v"])).max(initial=0)
    tol = bound * (u_w + 2 * ds[..., None] + 2.0 ** -18) + u_out * np.abs(want) + small * (1 + u_out) + 2.0 ** -24
    got = out.cpu().double().numpy()
    bad = np.argwhere(~(np.abs(got - want) <= tol))
    assert not len(bad), (len(bad), bad[0], got[tuple(bad[0])], want[tuple(bad[0])], tol[tuple(bad[0])])
    gl = lse.cpu().double().numpy()
    none = np.isinf(wlse)
    assert (gl[none] == -np.inf).all()
    assert (np.abs(gl[~none] - wlse[~none]) <= ds[~none] + 2.0 ** -18 * (1 + np.abs(wlse[~none]))).all()


CASES = [
    # sizes, prefix, suffix, T, Hq, Hkv, page
    ([1], [1], [1], 1, 1, 1, 16),
    ([1], [0], [1], 1, 4, 2, 16),
    ([2], [5], [0, 3], 1, 4, 1, 16),
    ([3, 1, 2], [17, 64, 130], [1, 16, 33, 64, 65, 200], 1, 8, 2, 16),
    ([8], [300], [20] * 8, 1, 12, 2, 16),
    ([4, 0, 5], [129, 7, 0], [31, 0, 1, 63, 128, 257, 2, 90, 300], 1, 7, 1, 32),
    ([5], [1000], [700, 3, 64, 5, 1], 1, 14, 2, 64),
    ([2, 3], [70, 513], [9, 40, 5, 129, 66], 5, 8, 2, 16),
    ([3], [40], [3, 8, 150], 8, 6, 2, 128),
    ([17], [260], list(range(17)), 1, 8, 2, 16),
    ([40, 3], [500, 90], [30] * 43, 2, 16, 2, 64),
    ([70], [333], [12] * 70, 1, 20, 4, 32),
    ([2], [9], [3, 77], 3, 40, 1, 16),
]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,cache", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, F8), (torch.float16, F8)])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_over_shared_and_own_keys(build, case, dtype, cache, D):
    sizes, prefix, suffix, T, Hq, Hkv, page = CASES[case]
    t, h = make(sizes, prefix, suffix, T, Hq, Hkv, D, dtype, cache, page, 100 * case + D)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = call(t, D ** -0.5, status=status)
    assert int(status) == 0
    check(t, h, D ** -0.5, out, lse)


@pytest.mark.parametrize("dtype,cache,D,Hq,Hkv,T", [(torch.bfloat16, torch.bfloat16, 128, 8, 2, 4), (torch.float16, F8, 64, 6, 1, 7), (torch.bfloat16, torch.bfloat16, 64, 32, 1, 5)])
def test_ragged_queries_empty_rows_and_strides(build, dtype, cache, D, Hq, Hkv, T):
    """Fewer queries than slots, none at all, more queries than own tokens (their first see no own token), rollouts beyond the
    last group, no prompt, rows cut out of wider ones on both sides."""
    sizes = [3, 2, 4]
    suffix = [5, 1, 80, 0, 33, 2, 64, 65, 3, 10, 11]
    q_len = [T, 1, 0, 2, T, 3, 1, T, 2, T, 1]
    t, h = make(sizes, [0, 19, 128], suffix, T, Hq, Hkv, D, dtype, cache, 16, 7, q_len=q_len, extra_rollouts=2, stride_extra=24)
    R = len(suffix)
    wide = torch.full((R, T, Hq * D + 8), 3.0, dtype=dtype, device=DEV)
    out = wide[..., :Hq * D].unflatten(2, (Hq, D))
    got, lse = call(t, 0.11, out=out)
    check(t, h, 0.11, got, lse)
    assert (wide[..., Hq * D:] == 3.0).all()
    assert (out[9:] == 0).all() and (lse[9:] == -math.inf).all()          # beyond the last group
    assert (out[2] == 0).all() and (lse[2] == -math.inf).all()            # no queries
    assert (out[3, 2:] == 0).all()


@pytest.mark.parametrize("D,dtype", [(64, torch.bfloat16), (128, torch.float16)])
def test_many_short_items_of_many_rows(build, D, dtype):
    """Drafts and many heads to a cache head make each rollout's own keys an item of many rows; hundreds of them, one or a few
    tiles long, follow each other on every multiprocessor."""
    rng = np.random.default_rng(D)
    R = 130
    suffix = rng.integers(3, 450, R)
    suffix[::9] = rng.integers(3, 60, len(suffix[::9]))
    t, h = make([70, 60], [130, 700], suffix, 3, 64, 4, D, dtype, dtype, 16, 21, q_len=rng.integers(1, 4, R))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = call(t, D ** -0.5, status=status)
    assert int(status) == 0
    check(t, h, D ** -0.5, out, lse)


def test_steps_follow_each_other_without_waiting(build):
    """Lengths, queries and caches change between calls on one stream that nothing waits between; the second of two states
    shares the first one's workspace."""
    hora = _hora()
    a, ha = make([6, 3], [300, 40], [50, 3, 20, 77, 8, 16, 5, 9, 100], 1, 8, 2, 128, torch.bfloat16, torch.bfloat16, 16, 31, garbage=False)
    b, hb = make([40], [900], [33] * 40, 1, 8, 2, 128, torch.bfloat16, torch.bfloat16, 16, 32, garbage=False)
    size = max(hora.hora_group_attention_workspace_bytes(x["pl"].shape[0], x["q"].shape[0], 1, 8, 2, 128) for x in (a, b))
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    scale, got = 128 ** -0.5, []
    for i in range(12):
        x, h = (a, ha) if i % 2 == 0 else (b, hb)
        x["sl"].sub_(1).clamp_(min=1)                          # the next call sees one key less of each rollout
        h["sl"] = np.maximum(h["sl"] - 1, 1)
        out, lse = torch.empty_like(x["q"]), torch.empty(x["q"].shape[:3], device=DEV)
        hora.hora_group_attention(x["q"], x["off"], None, scale, x["k"], x["v"], None, None, x["pp"], x["pl"], x["sp"], x["sl"], out, lse, ws)
        got.append((x, dict(h), out, lse))
    torch.cuda.synchronize()
    for x, h, out, lse in got:
        check(x, h, scale, out, lse)


@pytest.mark.parametrize("D,Hq,Hkv,T,dtype,cache,page", [(128, 32, 4, 2, torch.bfloat16, torch.bfloat16, 64), (64, 16, 2, 3, torch.float16, torch.float16, 16),
                                                           (128, 40, 8, 1, torch.float16, torch.float16, 128), (128, 16, 2, 2, torch.bfloat16, F8, 32)])
def test_large_groups_over_long_prompts(D, Hq, Hkv, T, dtype, cache, page):
    """Sizes at which the normal build takes the wide kernel, against plain 64-bit arithmetic on the device."""
    rng = np.random.default_rng(5)
    sizes = [90, 33, 1, 150]
    R = sum(sizes)
    plen = [2600, 1023, 640, 1409]
    t, h = make(sizes, plen, rng.integers(T, 90, R), T, Hq, Hkv, D, dtype, cache, page, 51)
    scale = D ** -0.5
    out, lse = call(t, scale)
    u_out = UNIT[dtype]
    u_w = 2.0 ** -11 if cache == F8 else u_out
    k, v, q = (torch.from_numpy(h[x]).to(DEV) for x in ("k", "v", "q"))
    for i in range(len(sizes)):
        for r in range(int(h["off"][i]), int(h["off"][i + 1])):
            def rows(pool, pages, n):
                return pool[torch.from_numpy(pages[:-(-n // page)].astype(np.int64)).to(DEV)].transpose(1, 2).reshape(-1, Hkv, D)[:n].transpose(0, 1)
            n = int(h["sl"][r])
            kk = torch.cat([rows(k, h["pp"][i], plen[i]), rows(k, h["sp"][r], n)], 1)
            vv = torch.cat([rows(v, h["pp"][i], plen[i]), rows(v, h["sp"][r], n)], 1)
            qq = q[r].reshape(T, Hkv, Hq // Hkv, D).transpose(0, 1).reshape(Hkv, -1, D)              # [Hkv, T * g, D]
            z = scale * (qq @ kk.transpose(1, 2))
            seen = plen[i] + n - T + 1 + torch.arange(T, device=DEV)
            hidden = torch.arange(kk.shape[1], device=DEV) >= seen[:, None]
            z = z.reshape(Hkv, T, Hq // Hkv, -1).masked_fill(hidden[None, :, None, :], -math.inf).reshape(Hkv, T * (Hq // Hkv), -1)
            e = torch.logsumexp(z, -1, keepdim=True)
            w = torch.exp(z - e)
            back = lambda x: x.reshape(Hkv, T, Hq // Hkv, -1).transpose(0, 1).reshape(T, Hq, -1)  # noqa: E731
            want, bound, ds = back(w @ vv), back(w @ vv.abs()), D * 2.0 ** -23 * scale * (qq.abs() @ kk.abs().transpose(1, 2)).amax()
            small = 0.0 if u_w == 2.0 ** -8 else 2.0 ** -25 * kk.shape[1] * vv.abs().amax()
            tol = bound * (u_w + 2 * ds + 2.0 ** -18) + u_out * want.abs() + small * (1 + u_out) + 2.0 ** -24
            assert ((out[r].double() - want).abs() <= tol).all(), (i, r)
            assert ((lse[r].double() - back(e)[..., 0]).abs() <= ds + 2.0 ** -18 * (1 + back(e)[..., 0].abs())).all(), (i, r)


def test_long_lists_are_split_and_joined(build):
    """Few rows over many keys: every CTA gets a part of an item, so most of the result comes from joining."""
    for cache in (torch.bfloat16, F8):
        t, h = make([2], [5003], [2100, 1], 1, 4, 1, 128, torch.bfloat16, cache, 128, 11)
        out, lse = call(t, 128 ** -0.5)
        check(t, h, 128 ** -0.5, out, lse)


def test_scores_of_all_magnitudes(build):
    """Very peaked and very flat attention, and scores that grow and fall along the keys."""
    for q_scale in (1e-3, 30.0):
        t, h = make([3], [200], [100, 3, 50], 1, 8, 2, 128, torch.bfloat16, torch.bfloat16, 16, 12, q_scale=q_scale)
        out, lse = call(t, 128 ** -0.5)
        check(t, h, 128 ** -0.5, out, lse)


def test_twice_the_same_bits_and_workspace_contents_do_not_matter(build):
    t, _ = make([9, 30], [700, 65], [40] * 39, 2, 16, 4, 128, torch.bfloat16, torch.bfloat16, 32, 13)
    a, la = call(t, 0.09)
    b, lb = call(t, 0.09)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(la, lb)


def test_on_another_stream_and_through_the_object():
    hora = _hora()
    t, h = make([4, 4], [100, 30], [7] * 8, 1, 8, 2, 64, torch.float16, torch.float16, 16, 14)
    op = hora.GroupAttention(hora.PagedCache.over(t["k"], t["v"]), 8, 1, torch.float16, group_offsets=t["off"], prefix_pages=t["pp"],
                             prefix_len=t["pl"], suffix_pages=t["sp"], suffix_len=t["sl"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, lse = op.run(t["q"])
    side.synchronize()
    check(t, h, 64 ** -0.5, out, lse)


def test_thousands_of_small_groups(build):
    """More sequences than a thread of the plan keeps in registers, empty groups among them; a sample of the rollouts is checked."""
    rng = np.random.default_rng(8)
    sizes = rng.integers(0, 7, 1700)
    R = int(sizes.sum())
    assert R + 1700 > 4 * 1024
    t, h = make(sizes, rng.integers(0, 40, 1700), rng.integers(0, 50, R), 1, 3, 1, 64, torch.bfloat16, torch.bfloat16, 16, 61)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = call(t, 0.125, status=status)
    assert int(status) == 0
    group = np.repeat(np.arange(1700), sizes)
    for r in rng.permutation(R)[:80].tolist() + [0, R - 1]:
        i = group[r]
        k, v = (np.concatenate([pool[h["pp"][i][np.arange(h["pl"][i]) // 16], 0, np.arange(h["pl"][i]) % 16],
                                pool[h["sp"][r][np.arange(h["sl"][r]) // 16], 0, np.arange(h["sl"][r]) % 16]]) for pool in (h["k"], h["v"]))
        for x in range(3):
            want, wlse, bound, reach = orc.attention_query(h["q"][r, 0, x], k, v, 0.125)
            tol = bound * (2.0 ** -8 + 64 * 2.0 ** -22 * reach + 2.0 ** -18) + 2.0 ** -8 * np.abs(want) + 2.0 ** -24
            assert (np.abs(out[r, 0, x].double().cpu().numpy() - want) <= tol).all(), (r, x)
            got = float(lse[r, 0, x])
            assert got == wlse if math.isinf(wlse) else abs(got - wlse) <= 64 * 2.0 ** -23 * reach + 2.0 ** -18 * (1 + abs(wlse))


@pytest.mark.parametrize("cache", [torch.bfloat16, F8])
def test_pages_beyond_32_bit_offsets(cache):
    """Pools of more than 2^32 bytes and 2^31 elements: keys and values in the last pages, written, read back and attended to."""
    hora = _hora()
    D, Hkv, page, G, P = 128, 2, 64, 40, 500
    n_pages = (1 << 31) // (Hkv * page * D) + 40 if cache != F8 else (1 << 32) // (Hkv * page * D) + 40
    c = hora.PagedCache.empty(n_pages, page, Hkv, D, cache)
    g = torch.Generator(device=DEV).manual_seed(4)
    pages = n_pages - 1 - torch.arange(8, device=DEV)
    own = n_pages - 9 - torch.arange(G, device=DEV) % 20            # rollouts share pages here: they are only read
    at = torch.arange(P, device=DEV)
    k, v = (torch.randn(P, Hkv, D, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    slots = pages[at // page] * page + at % page
    c.write(k, v, slots)
    ko, vo = (torch.empty(P, Hkv, D, device=DEV) for _ in range(2))
    c.read(slots, ko, vo)
    if cache != F8:
        assert torch.equal(ko, k.float()) and torch.equal(vo, v.float())
    else:
        assert ((ko - k.float()).abs() <= k.float().abs() / 16 + 2.0 ** -12 * k.float().abs().amax(-1, keepdim=True)).all()
    ks, vs = (torch.randn(20 * page, Hkv, D, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    c.write(ks, vs, ((n_pages - 9 - torch.arange(20, device=DEV))[:, None] * page + torch.arange(page, device=DEV)).flatten())
    kso, vso = (torch.empty(20 * page, Hkv, D, device=DEV) for _ in range(2))
    c.read(((n_pages - 9 - torch.arange(20, device=DEV))[:, None] * page + torch.arange(page, device=DEV)).flatten(), kso, vso)
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    q = torch.randn(G, 1, 4, D, device=DEV, generator=g).to(torch.bfloat16)
    op = hora.GroupAttention(c, 4, 1, torch.bfloat16, group_offsets=torch.tensor([0, G], device=DEV), prefix_pages=i32(pages)[None].contiguous(), prefix_len=i32([P]),
                             suffix_pages=i32(own)[:, None].contiguous(), suffix_len=i32([page] * G))
    out, _ = op.run(q)
    r = torch.arange(G, device=DEV) % 20
    kk = torch.cat([ko.double().expand(G, P, Hkv, D), kso.double().reshape(20, page, Hkv, D)[r]], 1).repeat_interleave(2, 2)
    vv = torch.cat([vo.double().expand(G, P, Hkv, D), vso.double().reshape(20, page, Hkv, D)[r]], 1).repeat_interleave(2, 2)
    w = torch.softmax(torch.einsum("rhd,rnhd->rhn", q[:, 0].double(), kk) * D ** -0.5, -1)
    want, bound = torch.einsum("rhn,rnhd->rhd", w, vv), torch.einsum("rhn,rnhd->rhd", w, vv.abs())
    assert ((out[:, 0].double() - want).abs() <= 2.0 ** -8 * (bound + want.abs()) + 2.0 ** -12 * bound + 1e-6).all()


def test_values_that_are_out_of_range_are_reported_and_stay_in_bounds(build):
    """Lengths, counts, page numbers and offsets that cannot be: reported, clamped; the other rollouts' results stand."""
    hora = _hora()
    for what in ("page", "length", "negative", "offsets", "q_len"):
        t, h = make([2, 3], [50, 20], [8, 9, 30, 12, 1], 2, 4, 2, 64, torch.bfloat16, torch.bfloat16, 16, 15, q_len=[2, 1, 2, 2, 1], garbage=False)
        if what == "page":
            t["sp"][4, 0] = 10 ** 6
        elif what == "length":
            t["sl"][4] = 10 ** 6
            t["sp"].clamp_(min=0)
        elif what == "negative":
            t["sl"][4] = -5
        elif what == "q_len":
            t["q_len"][4] = 9
        else:
            t["off"][2] = 99
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out, lse = call(t, 0.1, status=status)
        assert int(status) == hora.ERR_INVALID_VALUE, what
        want = orc.group_attention(h["q"], h["off"], h["ql"], 0.1, h["k"], h["v"], h["pp"], h["pl"], h["sp"], h["sl"])[0]
        assert np.abs(out.cpu().double().numpy() - want)[:4].max() < 0.05, what
