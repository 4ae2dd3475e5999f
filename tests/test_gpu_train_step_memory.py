"""The differentiable calls of the training example leave nothing on the device behind once their results are dropped, without the help of
Python's collector of cycles."""
from __future__ import annotations

import gc
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_nothing_is_left_behind():
    import train_groups as tg
    T, Hq, Hkv, D = 300, 4, 2, 64
    leaf = lambda h: torch.randn(T, h, D, device="cuda").bfloat16().requires_grad_()  # noqa: E731
    q, k, v = leaf(Hq), leaf(Hkv), leaf(Hkv)
    w = [torch.ones(D, device="cuda", requires_grad=True) for _ in range(2)]
    pos = torch.arange(T, device="cuda", dtype=torch.int32)
    freq = 10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
    off, first = (torch.tensor(x, dtype=torch.int64, device="cuda") for x in ([0, 100, 180, 300], [0, 2]))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step():
        rq, rk = tg.rotate.apply(q, k, *w, pos, freq)
        out = tg.attend.apply(rq, rk, v, off, first, status)
        return torch.autograd.grad(out, (q, k, v, *w), torch.ones_like(out))

    step()
    torch.cuda.synchronize()
    gc.collect()
    before, enabled = torch.cuda.memory_allocated(), gc.isenabled()
    gc.disable()
    try:
        for _ in range(3):
            step()
        torch.cuda.synchronize()
        assert torch.cuda.memory_allocated() == before
    finally:
        if enabled:
            gc.enable()
    assert int(status) == 0
