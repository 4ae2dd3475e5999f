"""hora_kv_write / hora_kv_read with rows that are views of other tensors."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("H,D", [(2, 64), (5, 128)])
def test_one_token_cut_out_of_heads_that_lie_first(H, D):
    """[H, 1, D] transposed to [1, H, D], as a projection with its heads in front gives it for one token."""
    from paper_2605_07114_b200 import hora
    k, v = (torch.randn(H, 1, D, device="cuda").to(torch.bfloat16).transpose(0, 1) for _ in range(2))
    assert k.stride(0) == D
    c = hora.PagedCache.empty(2, 16, H, D)
    slot = torch.tensor([19], device="cuda")
    c.write(k, v, slot)
    ko, vo = (torch.zeros(H, 1, D, dtype=torch.bfloat16, device="cuda").transpose(0, 1) for _ in range(2))
    c.read(slot, ko, vo)
    assert torch.equal(ko, k) and torch.equal(vo, v)
    assert torch.equal(c.k[1, :, 3], k[0]) and torch.equal(c.v[1, :, 3], v[0])
