"""The operators together, as the example runs them: a step's attention is held against attention over keys and values
that are kept apart from the cache, and the lengths against the tokens made."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _example():
    import importlib.util
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location("decode_groups", os.path.join(root, "examples", "decode_groups.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype,drafts", [("e4m3", 3), ("bf16", 3), ("bf16", 0)])
def test_example_runs_from_allocation_to_advantages(dtype, drafts):
    got = _example().run(prompts=7, steps=5, drafts=drafts, dtype=dtype, seed=3)
    assert got["status"] == 0
    R = got["R"]
    assert int(got["group_offsets"][-1]) == R == 7 * 32
    texts = torch.stack(got["texts"])                                # [steps, R, T]
    made = (texts >= 0).sum((0, 2))
    assert torch.equal(made.to(torch.int32), got["own_len"])
    assert int(texts.max()) < 997 and ((texts >= 0).sum(2) >= 1).all()
    assert torch.isfinite(got["adv"]).all() and torch.isfinite(got["target"]).all()
    if drafts:
        assert (texts[:, :, 1] >= 0).any()                           # some drafts are accepted


def test_a_step_of_the_layer_equals_dense_attention():
    """New tokens written and attended to as in the example, against attention over the same keys and values held densely in
    64 bits (bf16 cache: the cached values are the inputs)."""
    from paper_2605_07114_b200 import hora
    dev, g = "cuda", torch.Generator(device="cuda").manual_seed(1)
    N, G, P, T, Hq, Hkv, D, page = 3, 5, 70, 3, 8, 2, 64, 16
    R = N * G
    per_p, per_r = -(-P // page), 2
    pp = torch.randperm(N * per_p + R * per_r, device=dev, generator=g).to(torch.int32)
    prefix, suffix = pp[:N * per_p].reshape(N, per_p).contiguous(), pp[N * per_p:].reshape(R, per_r).contiguous()
    cache = hora.PagedCache.empty(N * per_p + R * per_r, page, Hkv, D, torch.bfloat16)
    new = lambda *s: torch.randn(*s, device=dev, generator=g).to(torch.bfloat16)  # noqa: E731
    at = torch.arange(P, device=dev)
    kp, vp = new(N, P, Hkv, D), new(N, P, Hkv, D)
    cache.write(kp.flatten(0, 1), vp.flatten(0, 1), (prefix.long()[:, at // page] * page + at % page).flatten())
    own = torch.zeros(R, dtype=torch.int32, device=dev)
    op = hora.GroupAttention(cache, Hq, T, torch.bfloat16, group_offsets=torch.arange(0, R + 1, G, device=dev), prefix_pages=prefix,
                             prefix_len=torch.full((N,), P, dtype=torch.int32, device=dev), suffix_pages=suffix, suffix_len=own)
    ks, vs = torch.zeros(R, 0, Hkv, D, device=dev, dtype=torch.float64), torch.zeros(R, 0, Hkv, D, device=dev, dtype=torch.float64)
    for step in range(4):
        k, v, q = new(R, T, Hkv, D), new(R, T, Hkv, D), new(R, T, Hq, D)
        place = own.long()[:, None] + torch.arange(T, device=dev)
        cache.write(k.flatten(0, 1), v.flatten(0, 1), (suffix.long().gather(1, place // page) * page + place % page).flatten())
        own += T
        ks, vs = torch.cat([ks, k.double()], 1), torch.cat([vs, v.double()], 1)
        out, _ = op.run(q)
        kk = torch.cat([kp.double().repeat_interleave(G, 0), ks], 1).repeat_interleave(Hq // Hkv, 2)
        vv = torch.cat([vp.double().repeat_interleave(G, 0), vs], 1).repeat_interleave(Hq // Hkv, 2)
        z = torch.einsum("rthd,rnhd->rhtn", q.double(), kk) * D ** -0.5
        seen = kk.shape[1] - T + torch.arange(T, device=dev)
        w = torch.softmax(z.masked_fill(torch.arange(kk.shape[1], device=dev) > seen[:, None], float("-inf")), -1)
        want, bound = torch.einsum("rhtn,rnhd->rthd", w, vv), torch.einsum("rhtn,rnhd->rthd", w, vv.abs())
        assert ((out.double() - want).abs() <= 2.0 ** -8 * (bound + want.abs()) + 2.0 ** -12 * bound + 1e-6).all(), step
