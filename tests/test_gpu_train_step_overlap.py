"""hora_packed_attention over sequences that overlap so much that their tiles are far more than tokens and sequences allow for: reported, and
nothing is written, neither outputs nor anything around the workspace."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV, PATTERN, MARGIN = "cuda", 0xA5, 1 << 20


@pytest.fixture(autouse=True, scope="module")
def gigabytes_are_given_back():
    yield
    torch.cuda.empty_cache()


def guarded(nbytes):
    """A buffer of bytes, and the larger one around it, all of the pattern."""
    around = torch.full((nbytes + 2 * MARGIN,), PATTERN, dtype=torch.uint8, device=DEV)
    return around[MARGIN:MARGIN + nbytes], around


def surroundings_intact(around):
    return bool((around[:MARGIN] == PATTERN).all()) and bool((around[-MARGIN:] == PATTERN).all())


@pytest.mark.parametrize("T,S,Hq,Hkv,causal", [
    (4000, 200, 8, 2, True),             # a few times as many tiles as there are places
    (4000, 4000, 128, 1, False),
    (131072, 65536, 128, 1, True),       # 2^31 tiles and more
])
def test_far_more_tiles_than_tokens(T, S, Hq, Hkv, causal):
    from paper_2605_07114_b200 import hora
    D = 64
    off = torch.zeros(S + 1, dtype=torch.int64, device=DEV)
    off[1::2] = T                                            # 0, T, 0, T, ..: every second sequence is all of the tokens
    rows = lambda h: torch.zeros(T, h, D, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    q, k, v = rows(Hq), rows(Hkv), rows(Hkv)
    for backward in (False, True):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        ws, ws_around = guarded(hora.hora_packed_attention_workspace_bytes(T, S, Hq, Hkv, D, backward))
        lse, lse_around = guarded(T * Hq * 4)
        outs = [guarded(T * h * D * 2) for h in ((Hq, Hkv, Hkv) if backward else (Hq,))]
        new = [o.view(torch.bfloat16).view(T, -1, D) for o, _ in outs]
        if backward:
            hora.hora_packed_attention_backward(q, k, v, q, lse.view(torch.float32).view(T, Hq), q, off, None, 0.1, causal, *new, ws, status)
        else:
            hora.hora_packed_attention(q, k, v, off, None, 0.1, causal, new[0], lse.view(torch.float32).view(T, Hq), ws, status)
        torch.cuda.synchronize()
        assert int(status) == 2
        assert surroundings_intact(ws_around)
        for _, around in [(lse, lse_around)] + outs:
            assert bool((around == PATTERN).all())
