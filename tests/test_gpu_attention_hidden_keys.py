"""hora_group_attention: what keys that a query does not see, and scores that are not finite, do to its result.  Eight or more queries to a key
and more than a hundred rows to a rollout's own keys, so that the checked build takes the wide kernel; every place of a key in a tile."""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda"


@pytest.fixture(params=["normal", "checked"])
def hora(request):
    from paper_2605_07114_b200 import build as b, hora
    if request.param == "checked":
        hora.use_library(b.build(checked=True))
        assert hora.hora_checked_violation() == 0
    yield hora
    left = hora.hora_checked_violation() if request.param == "checked" else 0
    hora.use_library(None)
    assert left == 0, f"index check failed: file {left >> 20}, line {left & 0xFFFFF}"


def attend(hora, q, k, v, own_len, prompt_len=0, prompt_page=0):
    """Rollout r has the first own_len[r] keys of pages 8 r .. 8 r + 7; the prompt those of page prompt_page."""
    R, T, Hq, D = q.shape
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    op = hora.GroupAttention(hora.PagedCache.over(k, v), Hq, T, q.dtype, group_offsets=torch.tensor([0, R], device=DEV), prefix_pages=i32([[prompt_page]]),
                             prefix_len=i32([prompt_len]), suffix_pages=torch.arange(8 * R, dtype=torch.int32, device=DEV).reshape(R, 8), suffix_len=i32(own_len))
    out, lse = op.run(q)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 120])
def test_a_hidden_draft_has_no_weight_at_all(hora, D, size):
    """The last key of each rollout is seen by its last query alone.  Whatever its values, the other queries get the same bits."""
    g = torch.Generator(device=DEV).manual_seed(D)
    R, T, Hq, page = 80, 2, 64, 16
    q = torch.randn(R, T, Hq, D, device=DEV, generator=g).to(torch.bfloat16)
    k, v = (torch.randn(8 * R, 1, page, D, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    own = 2 + np.arange(R)                                  # the hidden key is at every place of a tile of 64, and in the second one
    last = torch.as_tensor(own - 1, device=DEV)
    r = torch.arange(R, device=DEV)
    v[8 * r + last // page, 0, last % page] = 0.0
    want, want_lse = (x.clone() for x in attend(hora, q, k, v, own))
    v[8 * r + last // page, 0, last % page] = size
    got, got_lse = attend(hora, q, k, v, own)
    assert torch.equal(got[:, 0].view(torch.int16), want[:, 0].view(torch.int16)) and torch.equal(got_lse, want_lse)
    assert torch.isfinite(got.float()).all() and not torch.equal(got[:, 1], want[:, 1])


@pytest.mark.parametrize("D", [64, 128])
def test_a_score_beyond_fp32_makes_its_row_nan_at_every_place(hora, D):
    R, Hq, page = 66, 128, 16
    q = torch.zeros(R, 1, Hq, D, dtype=torch.bfloat16, device=DEV)
    q[:, :, ::2] = 2.0 ** 60                                # every other head
    k = torch.zeros(8 * R, 1, page, D, dtype=torch.bfloat16, device=DEV)
    v = torch.ones_like(k)
    at, r = torch.arange(R, device=DEV), torch.arange(R, device=DEV)
    k[8 * r + at // page, 0, at % page] = 2.0 ** 70
    out, lse = attend(hora, q, k, v, np.full(R, 70))
    assert torch.isnan(out[:, :, ::2]).all() and torch.isnan(lse[:, :, ::2]).all()
    assert (out[:, :, 1::2] == 1.0).all() and torch.isfinite(lse[:, :, 1::2]).all()
