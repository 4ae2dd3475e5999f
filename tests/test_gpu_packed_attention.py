"""hora_packed_attention and its backward pass against the formulas in 64 bits, element by element, within bounds that count the roundings."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import packed as orc  # noqa: E402

DEV = "cuda"
STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}          # half the smallest number of the type
BF, HF = torch.bfloat16, torch.float16


def offsets(lengths, start=0):
    off = [start]
    for n in lengths:
        off.append(off[-1] + n)
    return off


def inputs(T, Hq, Hkv, D, dtype, seed=0, sharp=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(T, 2 * Hq + 2 * Hkv, D, device=DEV, generator=g)
    x[:, :Hq] *= sharp
    x = x.to(dtype)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:Hq + 2 * Hkv], x[:, Hq + 2 * Hkv:]       # q, k, v, dout: slices of one projection


def run(q, k, v, dout, off, groups=None, causal=True, scale=None, backward=True, status=None):
    from paper_2605_07114_b200 import hora
    T, Hq, D = q.shape
    i64 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int64, device=DEV)  # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device=DEV) if status is None else status
    op = hora.PackedAttention(i64(off), T, Hq, k.shape[1], D, q.dtype, group_offsets=i64(groups), causal=causal, sm_scale=scale, status_dev=status, backward=backward)
    for t in (op.out, op.lse, op.dq, op.dk, op.dv):
        if t is not None:
            t.fill_(-7.0)
    out, lse = op.run(q, k, v)
    got = {"out": out, "lse": lse}
    if backward:
        got.update(zip(("dq", "dk", "dv"), op.backward(q, k, v, out, lse, dout)))
    torch.cuda.synchronize()
    return got, int(status)


def check(got, q, k, v, dout, off, groups=None, causal=True, scale=None):
    want, tol = orc.packed_attention(q, k, v, off, groups, causal, scale, dout if "dq" in got else None, STEP[q.dtype], TINY[q.dtype])
    for name, x in got.items():
        inside = x[off[0]:off[-1]].double()
        w, t = want[name][off[0]:off[-1]], tol[name][off[0]:off[-1]]
        assert torch.isfinite(inside).all(), name
        worst = float(((inside - w).abs() / (t + 1e-30)).max()) if inside.numel() else 0.0
        assert worst <= 1.0, f"{name}: {worst:.2f} of the bound"
        assert bool((x[:off[0]] == -7).all()) and bool((x[off[-1]:] == -7).all()), f"{name}: rows of no sequence were written"


SHAPES = [
    # lengths, Hq, Hkv, D, dtype, causal
    ([1], 1, 1, 128, BF, True),
    ([1, 1, 0, 2, 0], 4, 2, 64, HF, True),
    ([5], 12, 2, 128, BF, True),
    ([211], 12, 2, 128, BF, True),
    ([128, 256, 127, 129, 1], 4, 4, 128, BF, True),
    ([128, 256, 127, 129, 1], 4, 4, 128, HF, False),
    ([300, 17, 511], 28, 4, 128, BF, True),
    ([300, 17, 511], 10, 2, 64, BF, True),
    ([77, 513, 1, 33], 24, 2, 64, HF, True),
    ([77, 513, 1, 33], 6, 2, 128, HF, False),
    ([640, 3], 71, 1, 64, BF, True),
    ([130, 259], 28, 1, 128, HF, True),
    ([1500], 8, 1, 128, BF, True),
    ([1333, 700], 3, 3, 64, BF, False),
    ([70, 2], 128, 1, 64, BF, True),
    ([130, 40], 200, 1, 128, HF, True),
    ([95, 300], 48, 1, 128, BF, False),
]


@pytest.mark.parametrize("lengths,Hq,Hkv,D,dtype,causal", SHAPES)
def test_sequences(lengths, Hq, Hkv, D, dtype, causal):
    off = offsets(lengths)
    x = inputs(off[-1], Hq, Hkv, D, dtype)
    got, status = run(*x, off, causal=causal)
    assert status == 0
    check(got, *x, off, causal=causal)


GROUPS = [
    # lengths of each group: the prompt, then its rollouts
    ([[5, 3]], 4, 2, 64, BF, True),
    ([[211, 103, 1, 77, 200, 0, 13], [128, 5, 256]], 12, 2, 128, BF, True),
    ([[211, 103, 1, 77, 200, 0, 13], [128, 5, 256]], 12, 2, 64, HF, True),
    ([[300] + [150] * 20, [17, 33], [0, 9, 8], [64]], 28, 4, 128, BF, True),
    ([[129, 127, 128, 130], [1, 1, 1]], 6, 6, 128, HF, False),
    ([[40, 600, 3], [513, 2, 2]], 5, 1, 64, BF, False),
]


@pytest.mark.parametrize("groups,Hq,Hkv,D,dtype,causal", GROUPS)
def test_groups(groups, Hq, Hkv, D, dtype, causal):
    off, first = offsets([n for g in groups for n in g]), offsets([len(g) - 1 for g in groups])
    x = inputs(off[-1], Hq, Hkv, D, dtype, 1)
    got, status = run(*x, off, first, causal)
    assert status == 0
    check(got, *x, off, first, causal)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
def test_tokens_of_no_sequence_may_hold_anything(dtype, D):
    off = offsets([50, 0, 200, 131], 37)
    x = inputs(off[-1] + 90, 12, 4, D, dtype, 2)
    whole = [t.clone() for t in x]
    for t in whole:
        t[:37] = float("nan")
        t[off[-1]:] = float("inf")
        t[off[-1] + 3:off[-1] + 60] = float("nan")
    got, status = run(*whole, off)
    assert status == 0
    check(got, *x, off)


def test_a_sequence_with_nan_leaves_the_others_alone():
    off = offsets([150, 61, 200])
    x = inputs(off[-1], 8, 2, 128, BF, 3)
    clean, _ = run(*x, off)
    spoilt = [t.clone() for t in x]
    for t in spoilt:
        t[off[1]:off[2]] = float("nan")
    got, _ = run(*spoilt, off)
    for name in got:
        assert torch.equal(got[name][:off[1]], clean[name][:off[1]]) and torch.equal(got[name][off[2]:], clean[name][off[2]:]), name
        assert torch.isnan(got[name][off[1]:off[2]]).any()


@pytest.mark.parametrize("scale,sharp", [(0.001, 1.0), (1.0, 4.0), (0.0883, 40.0)])
def test_flat_and_sharp_scores(scale, sharp):
    off = offsets([400, 260])
    x = inputs(off[-1], 4, 2, 128, BF, 4, sharp)
    got, status = run(*x, off, scale=scale)
    assert status == 0
    check(got, *x, off, scale=scale)


@pytest.mark.parametrize("growth", [0.02, -0.02])
def test_a_maximum_that_keeps_moving(growth):
    """Scores that rise (or fall) along the keys: the reference of every row is raised again and again."""
    off = offsets([1100])
    q, k, v, dout = (t.clone() for t in inputs(off[-1], 2, 1, 128, BF, 5, 1.0))
    q[:] = q.abs() * 0.2 + 0.2
    k[:] = k * 0.2 + growth * torch.arange(off[-1], device=DEV)[:, None, None]
    got, status = run(q, k, v, dout, off)
    assert status == 0
    check(got, q, k, v, dout, off)


@pytest.mark.parametrize("size", [2.0 ** -14, 1.0, 2.0 ** 10])
def test_fp16_gradients_of_any_size(size):
    """Gradients of outputs far from one: those of scores are held relative to the largest, not in fp16 as they are."""
    off = offsets([300, 90])
    q, k, v, dout = inputs(off[-1], 4, 2, 128, HF, 6)
    dout = (dout.float() * size).to(HF)
    got, status = run(q, k, v, dout, off)
    assert status == 0
    check(got, q, k, v, dout, off)


def test_gradients_against_differences():
    """The loss sum(out * c) along a direction, by the library's own forward passes, in the library's own precision."""
    off, first = offsets([60, 30, 45, 20, 70]), [0, 2, 3]
    q, k, v, c = (t.float() for t in inputs(off[-1], 4, 2, 64, HF, 7))
    g = torch.Generator(device=DEV).manual_seed(8)
    got, _ = run(*(t.to(HF) for t in (q, k, v, c)), off, first)
    for i, name in enumerate(("dq", "dk", "dv")):
        x = [q, k, v]
        h = 0.25 * torch.randn(x[i].shape, device=DEV, generator=g)
        values, moved = [], []
        for sign in (1, -1):
            y = list(x)
            y[i] = (x[i] + sign * h).to(HF)
            moved.append(y[i].double())
            out, _ = run(*(t.to(HF) for t in y), c.to(HF), off, first, backward=False)
            values.append(float((out["out"].double() * c.to(HF).double()).sum()))
        slope, along = (values[0] - values[1]) / 2, float((got[name].double() * (moved[0] - moved[1]) / 2).sum())
        # two evaluations of sums of 900 * 64 terms rounded by 2^-11 of about 1/4 each, and a step whose third order is some percent
        assert abs(slope - along) <= 0.06 * abs(along) + 2.0, (name, slope, along)


def test_the_same_bits_every_time():
    groups = [[211, 103, 1, 77, 200, 0, 13], [128, 5, 256], [300] + [150] * 20]
    off, first = offsets([n for g in groups for n in g]), offsets([len(g) - 1 for g in groups])
    x = inputs(off[-1], 14, 2, 128, BF, 9)
    one, _ = run(*x, off, first)
    for _ in range(3):
        two, _ = run(*x, off, first)
        assert all(torch.equal(one[n], two[n]) for n in one)


@pytest.mark.parametrize("off,groups", [
    ([0, 40, 20, 100], None), ([0, 40, 400], None), ([-3, 40, 100], None), ([0, 100, 0, 100, 0, 100, 0, 100], None),
    ([0, 40, 60, 100], [0, 1]), ([0, 40, 60, 100], [0, 5]), ([0, 40, 60, 100], [1, 2]), ([0, 40, 60, 100], [0, 2, 1]), ([0, 40, 60, 100], [0, -1, 2]),
])
def test_bad_offsets_are_reported(off, groups):
    x = inputs(100, 4, 2, 64, BF, 10)
    assert run(*x, off, groups)[1] == 2


def test_rows_at_other_distances_and_given_outputs():
    from paper_2605_07114_b200 import hora
    off, T, Hq, Hkv, D = offsets([90, 170]), 260, 6, 2, 128
    x = inputs(T, Hq, Hkv, D, BF, 11)
    apart = []
    for i, t in enumerate(x):                            # 16, 24, .. elements more between the tokens, 16-byte aligned only
        width = t.shape[1] * D
        apart.append(torch.empty(T, width + 8 * (i + 2), dtype=BF, device=DEV)[:, 8:8 + width].unflatten(1, (t.shape[1], D)))
        apart[-1].copy_(t)
    i64 = torch.tensor(off, device=DEV)
    ws = torch.empty(hora.hora_packed_attention_workspace_bytes(T, 2, Hq, Hkv, D, True), dtype=torch.uint8, device=DEV)
    fused = torch.full((T, Hq + 2 * Hkv, D), 3.0, dtype=BF, device=DEV)
    out, lse = torch.empty(T, Hq + 1, D, dtype=BF, device=DEV)[:, 1:], torch.empty(T, Hq, device=DEV)
    dq, dk, dv = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    hora.hora_packed_attention(*apart[:3], i64, None, D ** -0.5, True, out, lse, ws)
    hora.hora_packed_attention_backward(*apart[:3], out, lse, apart[3], i64, None, D ** -0.5, True, dq, dk, dv, ws)
    torch.cuda.synchronize()
    check({"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, *x, off)
