"""hora_verify_drafts against the definition in exact integers and fractions: counts and tokens have to be equal."""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import decode as orc  # noqa: E402

DEV = "cuda"


def _hora():
    from paper_2605_07114_b200 import hora
    return hora


def draw(R, K, V, dtype, rows, seed, pad=0, spread=2.0, noise=0.6):
    rng = np.random.default_rng(seed)
    z = spread * rng.standard_normal((R, K + 1, V))

    def soft(x):
        e = np.exp(x - x.max(-1, keepdims=True))
        return torch.from_numpy(e / e.sum(-1, keepdims=True)).to(dtype)

    def strided(x):
        wide = torch.full((*x.shape[:2], V + pad), 2.0, dtype=dtype)
        wide[..., :V] = x
        return wide.to(DEV)[..., :V]

    target = soft(z)
    draft = soft(z[:, :K] + noise * rng.standard_normal((R, K, V))) if rows and K else None
    src = (target if draft is None else draft).double().numpy()
    tokens = np.zeros((R, K), np.int32)
    for r in range(R):
        for k in range(K):
            p = np.nan_to_num(src[r, k]) + 1e-12
            tokens[r, k] = rng.choice(V, p=p / p.sum())
    return dict(target=strided(target), draft=None if draft is None else strided(draft), tokens=torch.from_numpy(tokens).to(DEV),
                length=torch.from_numpy(rng.integers(0, K + 1, R).astype(np.int32)).to(DEV),
                u_accept=torch.rand(R, K, generator=torch.Generator().manual_seed(seed)).to(DEV),
                u_sample=torch.rand(R, generator=torch.Generator().manual_seed(seed + 1)).to(DEV))


def call(s, status=None):
    hora = _hora()
    R, K1, V = s["target"].shape
    n = torch.full((R,), -5, dtype=torch.int32, device=DEV)
    out = torch.full((R, K1), -5, dtype=torch.int32, device=DEV)
    hora.hora_verify_drafts(s["target"], s["draft"], s["tokens"], s["length"], R, K1 - 1, V, s["u_accept"], s["u_sample"], n, out, status)
    torch.cuda.synchronize()
    return n.cpu().numpy(), out.cpu().numpy()


def expect(s):
    h = {k: None if x is None else x.cpu().double().numpy() if x.is_floating_point() else x.cpu().numpy() for k, x in s.items()}
    R, K1, _ = h["target"].shape
    n, out = [], []
    for r in range(R):
        length = K1 - 1 if h["length"] is None else int(h["length"][r])
        a, b = orc.verify(h["target"][r], None if h["draft"] is None else h["draft"][r], h["tokens"][r], length, h["u_accept"][r], h["u_sample"][r])
        n.append(a)
        out.append(b)
    return np.array(n, np.int32), np.array(out, np.int32)


@pytest.mark.parametrize("rows", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R,K,V,pad", [(1, 0, 1, 0), (3, 1, 1, 0), (5, 2, 2, 0), (40, 4, 37, 0), (33, 8, 513, 0), (64, 3, 1000, 24), (20, 5, 4099, 3), (17, 4, 4096, 0), (6, 4, 12345, 1), (9, 40, 70, 0)])
def test_counts_and_tokens_are_the_definitions(R, K, V, pad, dtype, rows):
    s = draw(R, K, V, dtype, rows, 17 * R + K, pad)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    n, out = call(s, status)
    en, eo = expect(s)
    np.testing.assert_array_equal(n, en)
    np.testing.assert_array_equal(out, eo)
    assert int(status) == 0


def test_all_lengths_given_by_default_and_the_ends_of_the_random_numbers():
    s = draw(64, 3, 700, torch.float32, True, 5)
    s["length"] = None
    for u in (0.0, 1.0 - 2.0 ** -24, 2.0 ** -24, 0.5):
        s["u_sample"].fill_(u)
        s["u_accept"][::2].fill_(u)
        n, out = call(s)
        en, eo = expect(s)
        np.testing.assert_array_equal(n, en)
        np.testing.assert_array_equal(out, eo)


def test_large_vocabulary():
    s = draw(3, 1, 151936, torch.float32, True, 6)
    n, out = call(s)
    en, eo = expect(s)
    np.testing.assert_array_equal(n, en)
    np.testing.assert_array_equal(out, eo)


def test_rows_with_little_in_them():
    """One certain token, a difference with nothing left of it (drawn from the target then), mass in the last place, equal weights."""
    V = 1030
    t = torch.zeros(4, 2, V)
    d = torch.zeros(4, 1, V)
    t[0, :, 700] = 1.0
    d[0, 0, 3] = 1.0
    t[1, :, :] = 1.0 / V                                     # refused, and the draft's row covers the target's: nothing is left
    d[1, 0, :] = 1.0 / V
    d[1, 0, 9] = 0.5
    t[2, :, V - 1] = 2.0 ** -38
    d[2, 0, 0] = 1.0
    t[3, :, :] = 2.0 ** -11
    d[3, 0, 5] = 1.0
    s = dict(target=t.to(DEV), draft=d.to(DEV), tokens=torch.tensor([[3], [9], [0], [5]], dtype=torch.int32, device=DEV), length=None,
             u_accept=torch.full((4, 1), 0.9999, device=DEV), u_sample=torch.tensor([0.3, 0.77, 0.999, 0.5], device=DEV))
    n, out = call(s)
    en, eo = expect(s)
    np.testing.assert_array_equal(n, en)
    np.testing.assert_array_equal(out, eo)
    assert out[0, 0] == 700 and out[2, 0] == V - 1


def test_values_that_are_out_of_range_are_reported():
    hora = _hora()
    for what in ("token", "length", "nan", "negative", "empty"):
        s = draw(6, 2, 300, torch.float32, True, 8)
        s["length"].fill_(2)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        if what == "token":
            s["tokens"][4, 0] = 300
        elif what == "length":
            s["length"][4] = 7
        elif what == "empty":
            s["target"][4] = 0
        else:
            s["target"][4, :, 11] = float("nan") if what == "nan" else -0.25
        n, out = call(s, status)
        assert int(status) == hora.ERR_INVALID_VALUE, what
        if what == "length":
            s["length"][4] = 2
        en, eo = expect(s)
        np.testing.assert_array_equal(n, en)
        np.testing.assert_array_equal(out, eo)
        if what == "empty":
            assert out[4, n[4]] == -1


def test_the_tokens_follow_the_target():
    """Speculative sampling leaves the target's distribution: frequencies of the first token over many draws, within five
    standard deviations of a binomial count."""
    V, R = 8, 60000
    g = torch.Generator(device=DEV).manual_seed(3)
    p = torch.softmax(torch.randn(V, device=DEV, generator=g), -1)
    q = torch.softmax(torch.randn(V, device=DEV, generator=g), -1)
    tokens = torch.multinomial(q, R, replacement=True, generator=g).to(torch.int32).unsqueeze(1)
    s = dict(target=p.expand(R, 2, V).contiguous(), draft=q.expand(R, 1, V).contiguous(), tokens=tokens, length=None,
             u_accept=torch.rand(R, 1, device=DEV, generator=g), u_sample=torch.rand(R, device=DEV, generator=g))
    n, out = call(s)
    got = np.bincount(out[:, 0], minlength=V)
    want = p.double().cpu().numpy() * R
    assert (np.abs(got - want) <= 5 * np.sqrt(want * (1 - want / R)) + 1).all()
