"""hora_group_attention with many query slots (a chunk of a prompt, many drafts), and with short lists of many rows at sizes at which the normal
build takes the wide kernel.  Tolerances are those of test_gpu_group_attention.py."""
from __future__ import annotations

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_group_attention import DEV, F8, UNIT, build, call, check, make  # noqa: E402,F401


@pytest.mark.parametrize("dtype,cache", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, F8)])
@pytest.mark.parametrize("T,Hq,Hkv,D", [(9, 4, 2, 64), (16, 2, 1, 128), (33, 4, 4, 64), (64, 8, 2, 128), (131, 3, 1, 64)])
def test_many_query_slots(build, T, Hq, Hkv, D, dtype, cache):  # noqa: F811
    """As many queries as own tokens (a whole prompt), fewer, more (the first see no own key, and none at all without a prompt), one, none."""
    suffix = [T, 3 * T + 5, T // 2, 40, 1]
    t, h = make([3, 2], [0, 77], suffix, T, Hq, Hkv, D, dtype, cache, 16, T, q_len=[T, T, T, 1, 0])
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = call(t, D ** -0.5, status=status)
    assert int(status) == 0
    check(t, h, D ** -0.5, out, lse)


def test_the_most_query_slots(build):  # noqa: F811
    """T * Hq / Hkv at its limit."""
    t, h = make([1], [70], [500], 512, 8, 1, 64, torch.bfloat16, torch.bfloat16, 128, 3, q_len=[500])
    out, lse = call(t, 0.125)
    check(t, h, 0.125, out, lse)


@pytest.mark.parametrize("T,Hq,Hkv,D,dtype,longest", [(5, 32, 4, 64, torch.bfloat16, 130), (3, 44, 4, 128, torch.float16, 64), (2, 64, 2, 128, torch.bfloat16, 300),
                                                      (8, 40, 2, 64, torch.float16, 33)])
def test_short_lists_of_many_rows_at_size(T, Hq, Hkv, D, dtype, longest):
    """Hundreds of rollouts whose own keys, one or a few tiles of them, have 33 rows and more: enough of them for the wide kernel in the normal build."""
    rng = np.random.default_rng(longest)
    g = Hq // Hkv
    sizes = [250, 1, 349, 600]
    R = sum(sizes)
    own = np.maximum(rng.integers(1, longest + 1, R), 1)
    q_len = np.minimum(rng.integers(1, T + 1, R), own)
    prompt = np.array([100, 0, 333, 64])
    t, h = make(sizes, prompt, own, T, Hq, Hkv, D, dtype, dtype, 16, 4, q_len=q_len)
    keys, block = (16, 16) if D == 128 else (32, 24)        # of a narrow step: more than sixteen of them to each of twelve streams a multiprocessor
    steps = sum((np.ceil(n / keys) * np.ceil(x * T * g / block)).sum() * Hkv for n, x in ((prompt, np.array(sizes)), (own, 1)))
    assert T * g >= 33 and steps > 16 * 148 * 12
    scale = D ** -0.5
    out, lse = call(t, scale)
    u = UNIT[dtype]
    k, v, q = (torch.from_numpy(h[x]).to(DEV) for x in ("k", "v", "q"))

    def rows(pool, pages, n):
        return pool[torch.from_numpy(pages[:-(-n // 16)].astype(np.int64)).to(DEV)].transpose(1, 2).reshape(-1, Hkv, D)[:n].transpose(0, 1)

    for i in range(len(sizes)):
        n_p = int(h["pl"][i])
        kp, vp = (rows(x, h["pp"][i], n_p) for x in (k, v))
        for r in range(int(h["off"][i]), int(h["off"][i + 1])):
            n, ql = int(own[r]), int(q_len[r])
            kk, vv = torch.cat([kp, rows(k, h["sp"][r], n)], 1), torch.cat([vp, rows(v, h["sp"][r], n)], 1)
            z = scale * (q[r, :ql].reshape(ql, Hkv, g, D).permute(1, 0, 2, 3).reshape(Hkv, ql * g, D) @ kk.transpose(1, 2))
            ds = D * 2.0 ** -23 * scale * float((q[r, :ql].abs().amax() * kk.abs().amax(1).sum(-1).amax()))
            seen = n_p + n - ql + 1 + torch.arange(ql, device=DEV)
            z = z.reshape(Hkv, ql, g, -1).masked_fill(torch.arange(kk.shape[1], device=DEV) >= seen[:, None, None], -math.inf).reshape(Hkv, ql * g, -1)
            e = torch.logsumexp(z, -1, keepdim=True)
            w = torch.exp(z - e)
            back = lambda x: x.reshape(Hkv, ql, g, -1).permute(1, 0, 2, 3).reshape(ql, Hq, -1)  # noqa: E731
            want, bound, e = back(w @ vv), back(w @ vv.abs()), back(e)[..., 0]
            small = 0.0 if u == 2.0 ** -8 else 2.0 ** -25 * kk.shape[1] * vv.abs().amax()
            assert ((out[r, :ql].double() - want).abs() <= bound * (u + 2 * ds + 2.0 ** -18) + u * want.abs() + small * (1 + u) + 2.0 ** -24).all(), r
            assert ((lse[r, :ql].double() - e).abs() <= ds + 2.0 ** -18 * (1 + e.abs())).all(), r
            assert (out[r, ql:] == 0).all() and (lse[r, ql:] == -math.inf).all()
