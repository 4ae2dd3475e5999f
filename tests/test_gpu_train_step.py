"""The operators of prompts and training steps together, as a layer uses them: one after the other, replayed from a graph, on several streams, dropped
with work in flight, at many sequences and beyond 32-bit offsets, and through the checked build."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import packed as orc  # noqa: E402
import test_gpu_packed_attention as tpa  # noqa: E402

DEV, BF, HF = "cuda", torch.bfloat16, torch.float16


def i64(x):
    return torch.tensor(x, dtype=torch.int64, device=DEV)


class Layer:
    """Queries, keys and values of a projection -> norm and rotation -> attention, and back."""

    def __init__(self, off, first, T, Hq, Hkv, D, dtype, seed=0):
        from paper_2605_07114_b200 import hora
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.Hq, self.Hkv, self.D, self.g = Hq, Hkv, D, g
        self.freq = 10000.0 ** (-torch.arange(0, D, 2, device=DEV, dtype=torch.float64) / D)
        self.w = [1 + 0.2 * torch.randn(D, device=DEV, generator=g) for _ in range(2)]
        self.rotation = hora.QkRotation(self.freq, D, q_weight=self.w[0], k_weight=self.w[1])
        self.off, self.first = i64(off), None if first is None else i64(first)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.attention = hora.PackedAttention(self.off, T, Hq, Hkv, D, dtype, group_offsets=self.first, status_dev=self.status, backward=True)
        self.qkv = torch.randn(T, Hq + 2 * Hkv, D, device=DEV, generator=g).to(dtype)
        self.dout = torch.randn(T, Hq, D, device=DEV, generator=g).to(dtype)
        self.positions = torch.randint(0, 4096, (T,), device=DEV, generator=g, dtype=torch.int32)
        self.qk = torch.empty(T, Hq + Hkv, D, device=DEV, dtype=dtype)
        self.d_qkv = torch.zeros_like(self.qkv)
        self.dw = [torch.zeros(D, device=DEV) for _ in range(2)]

    def step(self):
        Hq, n = self.Hq, self.Hq + self.Hkv
        q, k, v = self.qkv[:, :Hq], self.qkv[:, Hq:n], self.qkv[:, n:]
        rq, rk = self.qk[:, :Hq], self.qk[:, Hq:]
        self.rotation.run(q, k, self.positions, rq, rk)
        out, lse = self.attention.run(rq, rk, v)
        dq, dk, _ = self.attention.backward(rq, rk, v, out, lse, self.dout, dv=self.d_qkv[:, n:])
        self.rotation.backward(dq, dk, q, k, self.positions, self.d_qkv[:, :Hq], self.d_qkv[:, Hq:n], self.dw[0], self.dw[1])
        return out, lse

    def results(self):
        return [t.clone() for t in (self.attention.out, self.attention.lse, self.d_qkv, *self.dw)]

    def exact(self):
        """The same in 64 bits by automatic differentiation, from the values that the layer holds."""
        D, Hq, n = self.D, self.Hq, self.Hq + self.Hkv
        qkv = self.qkv.double().requires_grad_()
        w = [x.double().requires_grad_() for x in self.w]
        angle = (self.positions.double()[:, None] * self.freq)[:, None]
        c, s = torch.cos(angle), torch.sin(angle)

        def turn(x, w):
            z = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
            a, b = z[..., :D // 2], z[..., D // 2:]
            return torch.cat([a * c - b * s, a * s + b * c], -1)

        g = Hq // self.Hkv
        q, k, v = turn(qkv[:, :Hq], w[0]), turn(qkv[:, Hq:n], w[1]).repeat_interleave(g, 1), qkv[:, n:].repeat_interleave(g, 1)
        outs = []
        off, first = self.off.tolist(), None if self.first is None else self.first.tolist()
        for (a, b), shared in orc.sequences(off, first):
            at = torch.arange(a, b, device=DEV)
            if shared is not None:
                at = torch.cat([torch.arange(*shared, device=DEV), at])
            z = torch.einsum("thd,khd->htk", q[a:b], k[at]) * D ** -0.5
            z = z.masked_fill(at[None, :] > torch.arange(a, b, device=DEV)[:, None], float("-inf"))
            outs.append(torch.einsum("htk,khd->thd", torch.softmax(z, -1), v[at]))
        out = torch.cat(outs)
        (out * self.dout.double()).sum().backward()
        return out.detach(), qkv.grad, w[0].grad, w[1].grad


GROUPS = [[90, 40, 3, 77], [33, 0, 129, 64, 20]]


def grouped(groups=GROUPS):
    return tpa.offsets([n for g in groups for n in g]), tpa.offsets([len(g) - 1 for g in groups])


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [(HF, 6, 2, 64), (BF, 4, 4, 128)])
def test_a_layer_and_its_gradients(dtype, Hq, Hkv, D):
    off, first = grouped()
    layer = Layer(off, first, off[-1], Hq, Hkv, D, dtype)
    layer.step()
    torch.cuda.synchronize()
    assert int(layer.status) == 0
    out, d_qkv, dwq, dwk = layer.exact()
    # roundings on the way of a gradient, each of at most half a step of its value: queries, keys, weights, output, gradients of scores (that of
    # outputs is exact here), dq or dk, the result; in the 2-norm they add up to less than their number times one, and the sums' terms are
    # larger than the sums by what cancels, which doubles it at most at these sizes
    step = torch.finfo(dtype).eps / 2
    for got, want, roundings in ((layer.attention.out, out, 4), (layer.d_qkv, d_qkv, 14), (layer.dw[0], dwq, 14), (layer.dw[1], dwk, 14)):
        assert float((got.double() - want).norm() / want.norm()) <= roundings * step


def test_a_step_replayed_from_a_graph_with_other_contents():
    off, first = grouped()
    T = off[-1]
    layer, other = (Layer(off, first, T, 6, 2, 128, BF) for _ in range(2))
    layer.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step()
    g = torch.Generator(device=DEV).manual_seed(5)
    for groups in (GROUPS, [[100, 13, 20, 77], [3, 100, 59, 64, 20]], [[1, 110, 33, 66], [50, 90, 1, 1, 104]]):
        new_off, new_first = grouped(groups)
        assert new_off[-1] == T
        for x in (layer, other):
            x.off.copy_(i64(new_off))
        qkv = torch.randn(layer.qkv.shape, device=DEV, generator=g).to(BF)
        for x in (layer, other):
            x.qkv.copy_(qkv)
        graph.replay()
        other.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(layer.results(), other.results())) and int(layer.status) == 0


def test_two_graphs_of_one_object_one_after_the_other():
    """They share the workspace: replays on one stream follow each other."""
    off, first = grouped()
    layer = Layer(off, first, off[-1], 4, 2, 64, HF)
    layer.step()
    want = layer.results()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for x in graphs:
        with torch.cuda.graph(x):
            layer.step()
    for _ in range(3):
        for x in graphs:
            x.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(layer.results(), want))


def test_several_streams_at_once():
    off, first = grouped([[400, 300, 200, 100, 50]] * 4)
    layers = [Layer(off, first, off[-1], 8, 2, 128, BF, seed) for seed in range(3)]
    want = []
    for x in layers:
        x.step()
        torch.cuda.synchronize()
        want.append(x.results())
        for t in (x.attention.out, x.attention.lse, x.d_qkv, *x.dw):
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for x, s in zip(layers, streams):
            with torch.cuda.stream(s):
                x.step()
    torch.cuda.synchronize()
    for x, w in zip(layers, want):
        assert all(torch.equal(a, b) for a, b in zip(x.results(), w))


def test_objects_dropped_with_their_work_in_front():
    """The workspace of a dropped object is not handed on before its stream is through with it."""
    off, first = grouped([[400, 300, 200, 100, 50]] * 4)
    layer = Layer(off, first, off[-1], 8, 2, 128, BF)
    layer.step()
    want = layer.results()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(4):
        x = Layer(off, first, off[-1], 8, 2, 128, BF)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
            x.step()
        d_qkv, size = x.d_qkv, x.attention.workspace.numel()
        del x
        torch.full((size,), 255, dtype=torch.uint8, device=DEV)          # takes the memory if it has been handed on
        torch.cuda.synchronize()
        assert torch.equal(d_qkv, want[2])


@pytest.mark.parametrize("n", [1, 31, 300])
def test_rows_far_apart(n):
    """Offsets of elements beyond 32 bits: tokens 2^23 elements from each other, at the end of a buffer of gigabytes."""
    from paper_2605_07114_b200 import hora
    Hq, Hkv, D, stride = 4, 2, 64, 1 << 23
    room = torch.empty(300 * stride, dtype=BF, device=DEV)
    x = tpa.inputs(n, Hq, Hkv, D, BF, 21)
    views, at = [], 0
    for t in x + tuple(torch.zeros_like(t) for t in (x[0], x[0], x[1], x[2])):
        v = torch.as_strided(room, t.shape, (stride, D, 1), at)
        v.copy_(t)
        views.append(v)
        at += t.shape[1] * D
    q, k, v, dout, out, dq, dk, dv = views
    off, lse = i64([0, n]), torch.empty(n, Hq, device=DEV)
    ws = torch.empty(hora.hora_packed_attention_workspace_bytes(n, 1, Hq, Hkv, D, True), dtype=torch.uint8, device=DEV)
    hora.hora_packed_attention(q, k, v, off, None, D ** -0.5, True, out, lse, ws)
    hora.hora_packed_attention_backward(q, k, v, out, lse, dout, off, None, D ** -0.5, True, dq, dk, dv, ws)
    want, _ = tpa.run(*x, [0, n])
    torch.cuda.synchronize()
    for a, b in ((out, "out"), (lse, "lse"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
        assert torch.equal(a, want[b]), b
    freq = 10000.0 ** (-torch.arange(0, D, 2, device=DEV, dtype=torch.float64) / D)
    pos = torch.arange(n, device=DEV, dtype=torch.int32)
    hora.hora_qk_rotate(q, k, pos, freq, dq, dk)
    near = hora.QkRotation(freq, D).run(x[0].contiguous(), x[1].contiguous(), pos)
    assert torch.equal(dq, near[0]) and torch.equal(dk, near[1])


def test_nothing_to_do():
    from paper_2605_07114_b200 import hora
    for T, off in ((0, [0]), (0, [0, 0, 0]), (40, [0]), (40, [17, 17, 17])):
        x = tpa.inputs(T, 4, 2, 64, BF, 26)
        got, status = tpa.run(*x, off)
        assert status == 0 and all(bool((t == -7).all()) for t in got.values())


def test_overlapping_sequences_write_nothing_else():
    """Offsets that are not in order, with keys under so many queries that they are cut into parts: reported, and what is behind the tokens stays."""
    T = 2000
    x = tpa.inputs(T, 8, 2, 64, BF, 27)
    for off in ([0, T] * 40, [0, T, 0, 700, 0, T, 0, T, 100, T]):
        got, status = tpa.run(*x, off)
        assert status == 2


def test_thousands_of_short_sequences_and_groups():
    off = tpa.offsets([1 + i % 3 for i in range(5000)])
    x = tpa.inputs(off[-1], 2, 1, 64, BF, 22)
    got, status = tpa.run(*x, off)
    assert status == 0
    tpa.check(got, *x, off)
    groups = [[i % 4] + [1 + (i + r) % 3 for r in range(i % 3)] for i in range(4200)]        # more than the plan keeps in shared memory
    off, first = tpa.offsets([n for g in groups for n in g]), tpa.offsets([len(g) - 1 for g in groups])
    x = tpa.inputs(off[-1], 1, 1, 64, HF, 23)
    got, status = tpa.run(*x, off, first)
    assert status == 0
    tpa.check(got, *x, off, first)


def test_a_prompt_under_many_rollouts_is_cut_into_parts():
    groups = [[300] + [40 + i % 50 for i in range(150)]]
    off, first = grouped(groups)
    x = tpa.inputs(off[-1], 8, 2, 128, BF, 24)
    got, status = tpa.run(*x, off, first)
    assert status == 0
    tpa.check(got, *x, off, first)


def test_prompts_into_the_cache_and_their_attention_as_the_decode_step_has_it():
    """The last token of a packed prompt attends like a single query of hora_group_attention over the cache that the prompt was written to."""
    from paper_2605_07114_b200 import hora
    lengths, Hq, Hkv, D, page = [37, 200, 129], 8, 2, 128, 16
    off = tpa.offsets(lengths)
    T, N = off[-1], len(lengths)
    q, k, v, _ = tpa.inputs(T, Hq, Hkv, D, BF, 25)
    freq = 10000.0 ** (-torch.arange(0, D, 2, device=DEV, dtype=torch.float64) / D)
    pos = torch.cat([torch.arange(n, device=DEV) for n in lengths]).to(torch.int32)
    rq, rk = hora.QkRotation(freq, D).run(q, k, pos)
    out, lse = hora.PackedAttention(i64(off), T, Hq, Hkv, D, BF).run(rq, rk, v)
    kv = torch.cat([rk, v], 1)
    per = -(-max(lengths) // page)
    cache = hora.PagedCache.empty(N * per, page, Hkv, D, BF)
    pages = torch.randperm(N * per, device=DEV).to(torch.int32).reshape(N, per)
    seq = torch.repeat_interleave(torch.arange(N, device=DEV), i64(lengths))
    p = pos.long()
    cache.write(kv[:, :Hkv], kv[:, Hkv:], pages.long()[seq, p // page] * page + p % page)
    last = i64(off[1:]) - 1
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    step = hora.GroupAttention(cache, Hq, 1, BF, group_offsets=i64(list(range(N + 1))), prefix_pages=pages, prefix_len=i32(lengths), suffix_pages=pages[:, :1].contiguous(),
                               suffix_len=i32([0] * N))
    # a query that is not the last of its own keys sees none of them
    got, got_lse = step.run(rq[last][:, None].contiguous())
    torch.cuda.synchronize()
    # both within the weights' and the output's roundings of the same value
    assert float((got[:, 0].double() - out[last].double()).abs().max()) <= 4 * 2.0 ** -8 * float(v.abs().max())
    assert float((got_lse[:, 0] - lse[last]).abs().max()) <= 1e-4


def test_through_the_checked_build():
    from paper_2605_07114_b200 import build, hora
    path = build.build(checked=True)
    hora.use_library(path)
    try:
        assert hora.hora_checked_violation() == 0
        for shape in (([1, 1, 0, 2, 0], 4, 2, 64, HF, True), ([300, 17, 511], 28, 4, 128, BF, True), ([77, 513, 1, 33], 6, 2, 128, HF, False), ([640, 3], 71, 1, 64, BF, True)):
            tpa.test_sequences(*shape)
        for groups in tpa.GROUPS:
            tpa.test_groups(*groups)
        tpa.test_tokens_of_no_sequence_may_hold_anything(BF, 128)
        test_a_prompt_under_many_rollouts_is_cut_into_parts()
        for off, groups in (([0, 40, 20, 100], None), ([0, 100, 0, 100, 0, 100, 0, 100], None), ([0, 40, 60, 100], [0, 5]), ([0, 40, 60, 100], [0, -1, 2])):
            tpa.test_bad_offsets_are_reported(off, groups)
        left = hora.hora_checked_violation()
    finally:
        hora.use_library(None)
    assert left == 0, f"index check failed: file {left >> 20}, line {left & 0xFFFFF}"
