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


def test_a_slot_given_twice_leaves_the_others_alone():
    """What such a slot holds is open; all others hold their token, and nothing else is written."""
    from paper_2605_07114_b200 import hora
    n, H, D, page = 300, 3, 128, 32
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn(n, H, D, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    for dtype in (torch.float8_e4m3fn, torch.bfloat16):
        c, once = (hora.PagedCache.empty(12, page, H, D, dtype) for _ in range(2))
        pools = [x for x in (c.k, c.v, c.k_exp, c.v_exp, once.k, once.v, once.k_exp, once.v_exp) if x is not None]
        for x in pools:
            x.view(torch.uint8).zero_()
        slots = torch.randperm(12 * page, device="cuda", generator=g)[:n]
        twice = slots.clone()
        twice[200:250] = slots[7]                              # fifty tokens and one share a slot
        slots[200:250] = -1
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        c.write(k, v, twice, status)
        once.write(k, v, slots, status)
        assert int(status) == 0
        at = (slots[7] // page, slice(None), slots[7] % page)
        half = len(pools) // 2
        for x, y in zip(pools[:half], pools[half:]):
            x, y = x.view(torch.uint8), y.view(torch.uint8)
            x[at] = y[at] = 0
            assert torch.equal(x, y)
