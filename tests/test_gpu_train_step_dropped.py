"""QkRotation and PackedAttention dropped with their work in front of another stream, whatever the allocator holds: their own memory is
not handed on before that stream is through with it.  What the caller gave them the caller keeps."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_train_step import BF, DEV, Layer, grouped  # noqa: E402


@pytest.mark.parametrize("cached", [0, 1 << 30])
def test_the_objects_own_memory(cached):
    torch.cuda.empty_cache()
    off, first = grouped([[400, 300, 200, 100, 50]] * 4)
    layer = Layer(off, first, off[-1], 8, 2, 128, BF)
    layer.step()
    want = layer.results()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(4):
        if cached:                                           # one large block, which the object's memory is then cut from
            torch.empty(cached, dtype=torch.uint8, device=DEV)
        x = Layer(off, first, off[-1], 8, 2, 128, BF)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
            x.step()
        size = x.attention.workspace.numel()
        span = lambda t: (t.data_ptr(), t.data_ptr() + t.numel() * t.element_size())  # noqa: E731
        owned = [span(getattr(x.attention, n)) for n in ("workspace", "out", "lse", "dq", "dk", "dv")] + [span(x.rotation.workspace)]
        del x.attention, x.rotation
        taken = [torch.full((n,), 255, dtype=torch.uint8, device=DEV) for n in (size, size // 4, size // 16, 1 << 16)]
        early = not side.query()                             # else the stream is through with them, and they may be anybody's
        for lo, hi in map(span, taken):
            assert not early or all(hi <= a or b <= lo for a, b in owned)
        torch.cuda.synchronize()
        assert torch.equal(x.d_qkv, want[2]) and all(torch.equal(a, b) for a, b in zip(x.dw, want[3:]))
        del x, taken
    torch.cuda.empty_cache()
