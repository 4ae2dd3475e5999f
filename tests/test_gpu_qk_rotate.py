"""hora_qk_rotate and its backward pass against the formulas in 64 bits."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import packed as orc  # noqa: E402

DEV = "cuda"
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def make(n, Hq, Hk, D, rot, dtype, norm, seed=0, far=32768):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    x = r(n, Hq + 2 * Hk, D).to(dtype)
    w = [1 + 0.3 * r(D) if norm else None for _ in range(2)]
    freq = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot) if rot else None
    pos = torch.randint(-far, far, (n,), device=DEV, generator=g, dtype=torch.int32)
    return x[:, :Hq], x[:, Hq:Hq + Hk], pos, freq, w, r(n, Hq, D).to(dtype), r(n, Hk, D).to(dtype)


def near(name, got, want, size, dtype, ops):
    """One rounding to the type, and `ops` in 32 bits on terms of the given size."""
    tol = STEP[dtype] * want.abs() + ops * 2.0 ** -24 * size + TINY[dtype]
    worst = float(((got.double() - want).abs() / (tol + 1e-30)).max()) if got.numel() else 0.0
    assert worst <= 1.0, f"{name}: {worst:.2f} of the bound"


CASES = [
    # n, Hq, Hk, D, rot, dtype, pairs, norm
    (1, 1, 1, 128, 128, torch.bfloat16, False, True),
    (3, 12, 2, 128, 128, torch.bfloat16, False, True),
    (480, 28, 4, 128, 128, torch.bfloat16, False, True),
    (101, 7, 3, 64, 64, torch.float16, False, True),
    (101, 7, 3, 64, 64, torch.float16, True, False),
    (257, 5, 1, 64, 32, torch.float32, True, True),
    (257, 5, 1, 128, 48, torch.float32, False, True),
    (33, 40, 8, 128, 16, torch.bfloat16, False, False),
    (33, 2, 2, 64, 0, torch.float32, False, True),
    (20000, 3, 1, 64, 64, torch.bfloat16, False, True),
    (10007, 2, 1, 128, 64, torch.float16, True, True),
]


@pytest.mark.parametrize("n,Hq,Hk,D,rot,dtype,pairs,norm", CASES)
def test_both_directions(n, Hq, Hk, D, rot, dtype, pairs, norm):
    from paper_2605_07114_b200 import hora
    if rot == 0 and not norm:
        pytest.skip("nothing to do")
    q, k, pos, freq, (wq, wk), dyq, dyk = make(n, Hq, Hk, D, rot, dtype, norm)
    op = hora.QkRotation(freq, D, q_weight=wq, k_weight=wk, eps=1e-5, layout=hora.ROTATE_PAIRS if pairs else hora.ROTATE_HALVES)
    yq, yk = op.run(q, k, pos)
    dwq, dwk = (torch.full((D,), -7.0, device=DEV) if norm else None for _ in range(2))
    dxq, dxk = op.backward(dyq, dyk, q if norm else None, k if norm else None, pos, dq_weight=dwq, dk_weight=dwk)
    torch.cuda.synchronize()
    f = freq if freq is not None else torch.zeros(0, dtype=torch.float64, device=DEV)
    for name, x, w, dy, y, dx, dw in (("q", q, wq, dyq, yq, dxq, dwq), ("k", k, wk, dyk, yk, dxk, dwk)):
        want_y, want_dx, want_dw = orc.qk_rotate(x, pos, f, pairs, w, 1e-5, dy)
        # terms of a pair: both values, at most sqrt(2) of the larger; the sum of squares of D values, a root, products, and the cosine and sine
        # of an angle whose fraction of a turn has 2^-25 of rounding (2 pi times that of an angle)
        size = (x.double().abs().amax(-1, keepdim=True) if w is None else w.double().abs().amax() * x.double().abs().amax(-1, keepdim=True) / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + 1e-5))
        near(name, y, want_y, 2 * size, dtype, 24)
        back = dy.double().abs().amax(-1, keepdim=True) * 2
        if w is not None:
            r = 1 / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + 1e-5)
            top = x.double().abs().amax(-1, keepdim=True) * r
            near("d" + name, dx, want_dx, r * w.abs().max() * back * (1 + top * top), dtype, 48)
            # partial sums of up to some thousands of terms in 32 bits
            terms = n * x.shape[1]
            near("dw" + name, dw, want_dw, (top * back).sum().expand(D) / max(1, terms) * terms ** 0.5 * 16 + want_dw.abs(), torch.float32, 64)
        else:
            near("d" + name, dx, want_dx, back, dtype, 24)


def test_far_positions_keep_their_angles():
    from paper_2605_07114_b200 import hora
    n, D = 64, 128
    q, k, _, freq, _, _, _ = make(n, 2, 1, D, D, torch.float32, False, 1)
    pos = torch.cat([2 ** 31 - 1 - torch.arange(n // 2, device=DEV), -2 ** 31 + torch.arange(n // 2, device=DEV)]).to(torch.int32)
    yq, _ = hora.QkRotation(freq, D).run(q, k, pos)
    # 2^31 turns have lost 2^-23 of one in 64 bits
    near("q", yq, orc.qk_rotate(q, pos, freq, False), 2 * q.double().abs().amax(-1, keepdim=True), torch.float32, 24)


def test_in_place_one_side_and_slices():
    from paper_2605_07114_b200 import hora
    q, k, pos, freq, (wq, wk), dyq, dyk = make(77, 6, 2, 128, 128, torch.bfloat16, True, 2)
    op = hora.QkRotation(freq, 128, q_weight=wq, k_weight=wk)
    yq, yk = op.run(q, k, pos)
    fused = torch.cat([q, k, k], 1)
    a, b = fused[:, :6], fused[:, 6:8]
    op.run(a, b, pos, a, b)
    assert torch.equal(a, yq) and torch.equal(b, yk) and torch.equal(fused[:, 8:], k)
    assert torch.equal(op.run(None, k, pos)[1], yk) and torch.equal(op.run(q, None, pos)[0], yq)
    dq, dk = op.backward(dyq, dyk, q, k, pos)
    both = [dyq.clone(), dyk.clone()]
    op.backward(*both, q, k, pos, *both)
    assert torch.equal(both[0], dq) and torch.equal(both[1], dk)


def test_no_tokens_and_bits():
    from paper_2605_07114_b200 import hora
    q, k, pos, freq, (wq, wk), dyq, dyk = make(5003, 6, 2, 64, 64, torch.bfloat16, True, 3)
    op = hora.QkRotation(freq, 64, q_weight=wq, k_weight=wk)
    dw = [torch.full((64,), -7.0, device=DEV) for _ in range(4)]
    one = op.backward(dyq, dyk, q, k, pos, dq_weight=dw[0], dk_weight=dw[1])
    two = op.backward(dyq, dyk, q, k, pos, dq_weight=dw[2], dk_weight=dw[3])
    assert all(torch.equal(x, y) for x, y in zip(one, two)) and torch.equal(dw[0], dw[2]) and torch.equal(dw[1], dw[3])
    op.backward(dyq[:0], dyk[:0], q[:0], k[:0], pos[:0], dq_weight=dw[0], dk_weight=dw[1])
    assert not dw[0].any() and not dw[1].any()
    op.run(q[:0], k[:0], pos[:0])


def test_what_is_not_finite_stays_in_its_row_or_pair():
    from paper_2605_07114_b200 import hora
    q, k, pos, freq, (wq, wk), _, _ = make(16, 2, 1, 128, 64, torch.bfloat16, True, 4)
    spoilt = q.clone()
    spoilt[3, 1, 5] = float("inf")
    normed, plain = hora.QkRotation(freq, 128, q_weight=wq, k_weight=wk), hora.QkRotation(freq, 128)
    for op, touched in ((normed, slice(None)), (plain, [5, 37])):
        a, b = op.run(q, None, pos)[0], op.run(spoilt, None, pos)[0]
        same = (a == b)
        other = torch.ones_like(same)
        other[3, 1, touched] = False
        assert bool(same[other].all())
    spoilt = q.clone()
    spoilt[3, 1, 100] = float("inf")                     # a value that is not turned
    assert bool((plain.run(spoilt, None, pos)[0] == plain.run(q, None, pos)[0]).sum() == q.numel() - 1)
