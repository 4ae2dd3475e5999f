"""The weights' gradients of hora_qk_rotate_backward where lanes of a warp have no head left (a ragged number of tokens, heads cut into
chunks), with eps = 0 as well: what idle lanes compute has no say."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import packed as orc  # noqa: E402
import test_gpu_qk_rotate as tqr  # noqa: E402

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("n,Hq,Hk,D,dtype", [
    (1, 1, 1, 64, F32), (1, 5, 2, 128, BF), (3, 28, 4, 128, BF), (7, 9, 3, 64, HF), (101, 7, 1, 128, F32), (9473, 2, 1, 64, BF), (9475, 1, 1, 128, HF), (20011, 3, 2, 64, F32),
])
def test_idle_lanes_have_no_say(n, Hq, Hk, D, dtype, eps):
    from paper_2605_07114_b200 import hora
    q, k, pos, freq, (wq, wk), dyq, dyk = tqr.make(n, Hq, Hk, D, D, dtype, True, 7)
    op = hora.QkRotation(freq, D, q_weight=wq, k_weight=wk, eps=eps)
    dw = [torch.full((D,), -7.0, device="cuda") for _ in range(2)]
    dx = op.backward(dyq, dyk, q, k, pos, dq_weight=dw[0], dk_weight=dw[1])
    torch.cuda.synchronize()
    for x, w, dy, got_dx, got in ((q, wq, dyq, dx[0], dw[0]), (k, wk, dyk, dx[1], dw[1])):
        _, want_dx, want = orc.qk_rotate(x, pos, freq, False, w, eps, dy)
        # as in the tests of both directions: a row's terms are at most its largest normed value times sqrt(2) of its largest gradient, and
        # partial sums of a square root's growth hold up to some thousands of them in 32 bits
        r = 1 / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + eps)
        top, back = x.double().abs().amax(-1, keepdim=True) * r, 2 * dy.double().abs().amax(-1, keepdim=True)
        terms = n * x.shape[1]
        tqr.near("dw", got, want, (top * back).sum().expand(D) / terms * terms ** 0.5 * 16 + want.abs(), F32, 64)
        tqr.near("dx", got_dx, want_dx, r * w.abs().max() * back * (1 + top * top), dtype, 48)
