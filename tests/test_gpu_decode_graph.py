"""A decode step replayed from a CUDA graph: the same bits as the calls by themselves, with contents that change between the replays."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_a_step_replayed_from_a_graph(dtype):
    from paper_2605_07114_b200 import hora
    g = torch.Generator(device=DEV).manual_seed(6)
    sizes, T, Hq, Hkv, D, page, V = [5, 60, 3], 3, 16, 2, 64, 16, 1003
    R, N = sum(sizes), len(sizes)
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g).to(torch.bfloat16)  # noqa: E731
    table = torch.randperm(N * 20 + R * 4, device=DEV, generator=g).to(torch.int32)
    prefix, suffix = table[:N * 20].reshape(N, 20).contiguous(), table[N * 20:].reshape(R, 4).contiguous()
    cache, other = (hora.PagedCache.empty(N * 20 + R * 4, page, Hkv, D, dtype) for _ in range(2))
    at = torch.arange(320, device=DEV)
    k, v = normal(N * 320, Hkv, D), normal(N * 320, Hkv, D)
    for c in (cache, other):
        c.write(k, v, (prefix.long()[:, at // page] * page + at % page).flatten())
    own, own2 = i32([0] * R), i32([0] * R)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    args = dict(group_offsets=torch.tensor([0, 5, 65, 68], device=DEV), prefix_pages=prefix, prefix_len=i32([300, 170, 31]), suffix_pages=suffix, status_dev=status)
    op, op2 = (hora.GroupAttention(c, Hq, T, torch.bfloat16, suffix_len=n, **args) for c, n in ((cache, own), (other, own2)))
    k, v, q = (torch.zeros(R, T, h, D, dtype=torch.bfloat16, device=DEV) for h in (Hkv, Hkv, Hq))
    slots = torch.full((R * T,), -1, device=DEV)
    target, draft = torch.zeros(R, T, V, device=DEV), torch.zeros(R, T - 1, V, device=DEV)
    tokens, u, us = i32([[0] * (T - 1)] * R), torch.zeros(R, T - 1, device=DEV), torch.zeros(R, device=DEV)

    def step(c, o, n, made):
        c.write(k.flatten(0, 1), v.flatten(0, 1), slots, status)
        o.run(q)
        hora.hora_verify_drafts(target, draft, tokens, None, R, T - 1, V, u, us, n, made, status)

    outs = [(torch.zeros(R, dtype=torch.int32, device=DEV), torch.zeros(R, T, dtype=torch.int32, device=DEV)) for _ in range(2)]
    target.fill_(1.0 / V)
    draft.fill_(1.0 / V)
    step(cache, op, *outs[0])                               # slots are negative: nothing is stored
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, op, *outs[0])
    for _ in range(6):
        place = own.long()[:, None] + torch.arange(T, device=DEV)
        slots.copy_((suffix.long().gather(1, place // page) * page + place % page).flatten())
        for x in (k, v, q):
            x.copy_(normal(*x.shape))
        own += T
        own2.copy_(own)
        target.copy_(torch.softmax(2 * torch.randn(R, T, V, device=DEV, generator=g), -1))
        draft.copy_(torch.softmax(torch.log(target[:, :-1]) + 0.5 * torch.randn(R, T - 1, V, device=DEV, generator=g), -1))
        tokens.copy_(torch.multinomial(draft.flatten(0, 1), 1, generator=g).reshape(R, T - 1))
        u.copy_(torch.rand(R, T - 1, device=DEV, generator=g))
        us.copy_(torch.rand(R, device=DEV, generator=g))
        graph.replay()
        step(other, op2, *outs[1])
        assert torch.equal(op.out.view(torch.int16), op2.out.view(torch.int16)) and torch.equal(op.lse, op2.lse)
        filled = (slots // page, slice(None), slots % page)
        for a, b in ((cache.k, other.k), (cache.v, other.v)):
            assert torch.equal(a.view(torch.uint8)[filled], b.view(torch.uint8)[filled])
        for a, b in zip(*outs):
            assert torch.equal(a, b)
        own.copy_(own2 - T + outs[0][0] + 1)
    assert int(status) == 0 and int(own.min()) >= 6


def test_buffers_outlive_their_object_on_another_stream():
    """An object that is dropped while another stream still has its call in front of it: its memory is not given to anyone else before
    that.  The side stream is kept busy for a fraction of a second meanwhile."""
    from paper_2605_07114_b200 import hora
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    cache = hora.PagedCache.empty(8, 16, 2, 64)
    cache.k.normal_()
    cache.v.normal_()
    args = dict(group_offsets=torch.tensor([0, 3], device=DEV), prefix_pages=i32([[0, 1]]), prefix_len=i32([30]), suffix_pages=i32([[2], [3], [4]]), suffix_len=i32([5, 16, 1]))
    q = torch.randn(3, 1, 8, 64, device=DEV).to(torch.bfloat16)
    op = hora.GroupAttention(cache, 8, 1, torch.bfloat16, **args)
    want = op.run(q)[0].clone()
    out, size, at = torch.empty_like(q), op.workspace.numel(), op.workspace.data_ptr()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        op.run(q, out=out)
    del op
    taken = [torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(2)]
    assert not side.query() and all(t.data_ptr() != at for t in taken)
    side.synchronize()
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))
