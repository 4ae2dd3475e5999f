"""hora_verify_drafts with drafted tokens that lie outside the vocabulary (a padding token, -1): refused, reported, and the
token that follows is drawn from the target's whole row, whatever lies behind the row in memory."""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_verify_drafts import DEV, draw, expect  # noqa: E402


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


@pytest.mark.parametrize("rows", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V,token", [(300, 300), (300, 301), (300, 511), (300, 1023), (300, -1), (300, -2 ** 31), (300, 2 ** 31 - 1), (512, 512), (1024, 1024),
                                     (513, 1023), (4099, 4099), (4099, 4100)])
def test_a_token_outside_the_vocabulary_is_refused(hora, V, token, dtype, rows):
    """The row after the refused one holds 1.0 throughout: were it read, the weights' sum would be wrong by as much."""
    R, K = 7, 2
    s = draw(R, K, V, dtype, rows, 11)
    wide = torch.ones(R * (K + 1) * V + 2048, dtype=dtype, device=DEV)     # the last row has ones behind it too
    target = wide[:R * (K + 1) * V].view(R, K + 1, V)
    target.copy_(s["target"])
    target[:, 1:] = 1.0
    s["target"] = target
    s["length"].fill_(K)
    s["tokens"][:, 0] = token                                             # refused at once: row 0 is drawn from, row 1 lies behind it
    s["tokens"][R - 1, 0] = 0                                             # and for the last rollout at the end of the buffer
    s["target"][R - 1, 0, 0], s["u_accept"][R - 1, 0] = 1.0, 0.5
    s["target"][R - 1, 1] = 0.25
    s["tokens"][R - 1, 1] = token
    s["u_sample"][::2] = 0.999
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    n = torch.full((R,), -5, dtype=torch.int32, device=DEV)
    out = torch.full((R, K + 1), -5, dtype=torch.int32, device=DEV)
    hora.hora_verify_drafts(s["target"], s["draft"], s["tokens"], s["length"], R, K, V, s["u_accept"], s["u_sample"], n, out, status)
    torch.cuda.synchronize()
    en, eo = expect(s)
    np.testing.assert_array_equal(n.cpu().numpy(), en)
    np.testing.assert_array_equal(out.cpu().numpy(), eo)
    assert int(status) == hora.ERR_INVALID_VALUE
    assert ((out.cpu().numpy()[np.arange(R), en] >= 0) & (out.cpu().numpy()[np.arange(R), en] < V)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R,V,pad", [(1, 2, 0), (9, 37, 0), (33, 1000, 24), (20, 4099, 3), (700, 513, 1), (2, 50257, 0)])
def test_without_drafts_a_token_is_drawn_from_the_target(hora, R, V, pad, dtype):
    from test_gpu_verify_drafts import call
    s = draw(R, 0, V, dtype, False, R + V, pad)
    s["u_sample"][::3] = 1.0 - 2.0 ** -24
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    n, out = call(s, status)
    en, eo = expect(s)
    np.testing.assert_array_equal(n, en)
    np.testing.assert_array_equal(out, eo)
    assert int(status) == 0 and (n == 0).all()
