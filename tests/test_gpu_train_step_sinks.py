"""Rows with one dominant key whose value is zero: what they put out comes from weights that are small next to the largest, which fp16 has to
hold as well as the others."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import packed as orc  # noqa: E402
import test_gpu_packed_attention as tpa  # noqa: E402

BF, HF = torch.bfloat16, torch.float16


def with_sinks(off, at, Hq, Hkv, D, dtype, nats, seed=31):
    """Queries, keys, values, gradients of outputs; the tokens `at` are keys `nats` above the others' mean score, with values of zero."""
    q, k, v, dout = (t.clone() for t in tpa.inputs(off[-1], Hq, Hkv, D, dtype, seed, 1.0))
    q[..., 0], k[..., 0] = 8.0, 0.0
    v *= 64.0                                                # outputs in the type's normal range
    k[at] = 0.0
    k[at, :, 0] = nats * D ** 0.5 / 8.0
    v[at] = 0.0
    return q, k, v, dout


CASES = [
    # lengths (of groups: the prompt first), groups, Hq, Hkv, D, causal
    ([4000], None, 2, 1, 128, True),
    ([2500, 1300], None, 2, 2, 64, True),
    ([1500], None, 4, 1, 128, False),
    ([700, 900, 333, 1201], [0, 3], 2, 1, 128, True),
]


@pytest.mark.parametrize("dtype", [HF, BF])
@pytest.mark.parametrize("nats", [6.0, 12.0, 16.0, 18.0])
@pytest.mark.parametrize("lengths,groups,Hq,Hkv,D,causal", CASES)
def test_small_weights_keep_their_bits(lengths, groups, Hq, Hkv, D, causal, nats, dtype):
    off = tpa.offsets(lengths)
    at = off[:1] if groups else off[:-1]                     # the first token of a sequence, or of the prompt that all of them see
    x = with_sinks(off, at, Hq, Hkv, D, dtype, nats)
    got, status = tpa.run(*x, off, groups, causal, backward=False)
    assert status == 0
    # in fp16 weights are held times 2^7 or more relative to the largest: below 2^-14 they are off by half of the smallest number, 2^-25 by 2^-7 of it
    want, tol = orc.packed_attention(*x[:3], off, groups, causal, step=tpa.STEP[dtype], tiny=tpa.TINY[dtype] * 2.0 ** -7)
    for name, more in (("out", tpa.TINY[dtype]), ("lse", 0.0)):              # and the result by half of the type's smallest number
        worst = float(((got[name].double() - want[name]).abs() / (tol[name] + more + 1e-30)).max())
        assert worst <= 1.0, f"{name}: {worst:.2f} of the bound"


@pytest.mark.parametrize("nats", [12.0, 16.0])
def test_gradients(nats):
    off = tpa.offsets([1500, 333])
    x = with_sinks(off, off[:-1], 4, 2, 128, HF, nats)
    got, status = tpa.run(*x, off)
    assert status == 0
    tpa.check(got, *x, off)


def test_a_sink_that_comes_late():
    """The reference is raised by far, and the weights before it become small."""
    off = tpa.offsets([1100])
    for late in (64, 700, 1099):
        q, k, v, dout = with_sinks(off, [late], 2, 1, 128, HF, 14.0)
        got, status = tpa.run(q, k, v, dout, off, None, False, backward=False)
        assert status == 0
        want, tol = orc.packed_attention(q, k, v, off, None, False, step=tpa.STEP[HF], tiny=tpa.TINY[HF] * 2.0 ** -7)
        for name in ("out", "lse"):
            assert bool(((got[name].double() - want[name]).abs() <= tol[name] + tpa.TINY[HF]).all()), name


@pytest.mark.parametrize("dtype", [HF, BF])
def test_scores_of_tens_of_millions_stay_finite(dtype):
    """Scores whose fp32 rounding is as large as what lies between them: weights mean little there, but outputs are still means of values."""
    T, D = 192, 64
    v = tpa.inputs(T, 1, 1, D, dtype, 41)[2]
    q, k = (torch.zeros(T, 1, D, device="cuda", dtype=dtype) for _ in range(2))
    q[..., 0], k[..., 0], q[..., 1] = 8192.0, 8192.0, 1.0
    for growth in (0, 8, 16, 24, 40, 600):
        k[64:, :, 1], k[128:, :, 1] = growth, 2 * growth
        got, status = tpa.run(q, k, v, v, [0, T], None, False, 0.34657359, backward=False)      # 2^25 in units of log2
        assert status == 0
        out = got["out"].double()
        step = 1 + 4 * tpa.STEP[dtype]                       # of the weights, their sum's terms and the result
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(got["lse"]).all())
        assert bool((out <= v.double().amax(0).clamp_min(0) * step + 1e-3).all()) and bool((out >= v.double().amin(0).clamp_max(0) * step - 1e-3).all())
