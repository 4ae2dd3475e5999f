"""hora_kv_write / hora_kv_read against the definition: codes, scale bytes and values bit for bit."""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import decode as orc  # noqa: E402

DEV = "cuda"
F8 = torch.float8_e4m3fn


def _hora():
    from paper_2605_07114_b200 import hora
    return hora


def _rows(n, H, D, dtype, seed, stride_extra=0):
    """k, v [n, H, D] cut out of one wider row (a fused projection), with the magnitudes of very different rows in it."""
    rng = np.random.default_rng(seed)
    wide = torch.zeros(n, 2 * H * D + stride_extra, dtype=dtype)
    x = rng.standard_normal((n, 2, H, D)) * np.exp2(rng.integers(-12, 6, (n, 2, H, 1)))
    wide[:, :2 * H * D] = torch.from_numpy(x.reshape(n, -1)).to(dtype)
    wide = wide.to(DEV)
    return wide[:, :H * D].unflatten(1, (H, D)), wide[:, H * D:2 * H * D].unflatten(1, (H, D))


def _expected(x, cache_dtype):
    """(stored bits, scale bytes or None, values) of rows [n, H, D]."""
    if cache_dtype != F8:
        y = x.cpu().to(cache_dtype)
        return y.view(torch.int16).numpy(), None, y.double().numpy()
    xs = x.cpu().double().numpy()
    codes, exps = np.zeros(xs.shape, np.uint8), np.zeros(xs.shape[:2], np.uint8)
    for i in np.ndindex(xs.shape[:2]):
        codes[i], exps[i] = orc.quantise_row(xs[i])
    return codes, exps, orc.VALUES[codes] * np.exp2(exps.astype(np.float64) - 127)[..., None]


@pytest.mark.parametrize("n,H,D,page,dtype,cache,out", [
    (1, 1, 64, 16, torch.bfloat16, F8, torch.bfloat16),
    (1, 4, 128, 16, torch.float32, F8, torch.float32),
    (37, 3, 128, 16, torch.bfloat16, F8, torch.bfloat16),
    (67, 5, 64, 32, torch.float16, F8, torch.float32),
    (129, 8, 128, 64, torch.float32, F8, torch.float16),
    (200, 1, 128, 128, torch.bfloat16, torch.bfloat16, torch.float32),
    (33, 7, 64, 16, torch.float32, torch.bfloat16, torch.bfloat16),
    (50, 2, 128, 32, torch.float16, torch.float16, torch.float16),
    (21, 33, 64, 16, torch.bfloat16, F8, torch.float16),
])
@pytest.mark.parametrize("extra", [0, 24])
def test_rows_go_in_and_out_bit_for_bit(n, H, D, page, dtype, cache, out, extra):
    hora = _hora()
    k, v = _rows(n, H, D, dtype, n + H, extra)
    n_pages = n // page + 3
    rng = np.random.default_rng(n)
    slots = rng.permutation(n_pages * page)[:n].astype(np.int64)
    c = hora.PagedCache.empty(n_pages, page, H, D, cache)
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(0x5A)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    s = torch.from_numpy(slots).to(DEV)
    c.write(k, v, s, status)
    ko, vo = (torch.full((n, H, D), 7.0, dtype=out, device=DEV) for _ in range(2))
    c.read(s, ko, vo, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for x, pool, exps, got in ((k, c.k, c.k_exp, ko), (v, c.v, c.v_exp, vo)):
        bits, e, values = _expected(x, cache)
        raw = pool.view(torch.uint8 if cache == F8 else torch.int16).cpu().numpy()
        np.testing.assert_array_equal(raw[slots // page, :, slots % page], bits)
        if e is not None:
            np.testing.assert_array_equal(exps.cpu().numpy()[slots // page, :, slots % page], e)
        untouched = np.ones((n_pages, page), bool)
        untouched[slots // page, slots % page] = False
        rest = pool.view(torch.uint8).cpu().numpy().transpose(0, 2, 1, 3)[untouched]
        assert (rest == 0x5A).all(), "a slot that was not named was written"
        want = torch.from_numpy(values).to(out)
        assert torch.equal(got.cpu(), want)


def test_values_at_the_edges_of_the_format():
    """Zeros, the largest codes on both sides of a power of two, ties, subnormal codes, huge and tiny rows, infinities, NaN."""
    hora = _hora()
    D = 64
    rows = np.zeros((10, D), np.float32)
    rows[1, :4] = [448.0, -448.0, 447.9, 17.0]             # exactly the largest code: exponent 0
    rows[2, :4] = [448.0001, 16.5, 17.5, -0.0]             # just over it: exponent 1
    rows[3, :8] = [256.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 1.5 * 2.0 ** -9, -2.0 ** -11, 0.0625, 2.0 ** -6]
    rows[4, :3] = [3.0e38, 1.0e30, -3.4e38]
    rows[5, :3] = [1.0e-38, 1.0e-40, -2.0e-39]
    rows[6, :4] = [np.inf, 3.0, -np.inf, 1.0]
    rows[7, :4] = [np.nan, 5.0, -5.25, 0.1]
    rows[8, :] = np.nan
    rows[9, :2] = [np.inf, -np.inf]
    k = torch.from_numpy(rows).to(DEV).unsqueeze(1)
    c = hora.PagedCache.empty(1, 16, 1, D, F8)
    s = torch.arange(10, device=DEV)
    c.write(k, -k, s)
    ko, vo = (torch.empty(10, 1, D, device=DEV) for _ in range(2))
    c.read(s, ko, vo)
    for r in range(10):
        codes, e = orc.quantise_row(rows[r])
        assert int(c.k_exp[0, 0, r]) == e, r
        got = c.k.view(torch.uint8)[0, 0, r].cpu().numpy()
        nan = np.isnan(rows[r])
        np.testing.assert_array_equal(got[~nan], codes[~nan], err_msg=str(r))
        assert ((got[nan] & 0x7F) == 0x7F).all()
        np.testing.assert_array_equal(ko[r, 0].cpu().numpy(), (orc.VALUES[codes] * 2.0 ** (e - 127)).astype(np.float32))


def test_slots_that_are_not_stored():
    hora = _hora()
    n, H, D = 40, 2, 128
    k, v = _rows(n, H, D, torch.bfloat16, 3)
    c = hora.PagedCache.empty(2, 16, H, D, F8)
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(0x11)
    slots = torch.full((n,), -1, dtype=torch.int64)
    slots[5], slots[17] = 31, 0
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    c.write(k, v, slots.to(DEV), status)
    ko, vo = (torch.full((n, H, D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    c.read(slots.to(DEV), ko, vo, status)
    assert int(status) == 0
    raw = c.k.view(torch.uint8).cpu().numpy().transpose(0, 2, 1, 3).reshape(32, H, D)
    assert (raw[1:31] == 0x11).all() and not (raw[31] == 0x11).all() and not (raw[0] == 0x11).all()
    assert (ko[[i for i in range(n) if i not in (5, 17)]] == 0).all()
    # a slot beyond the cache: reported, skipped, read as zeros
    slots[7] = 32
    c.write(k, v, slots.to(DEV), status)
    assert int(status) == hora.ERR_INVALID_VALUE
    status.zero_()
    c.read(slots.to(DEV), ko, vo, status)
    assert int(status) == hora.ERR_INVALID_VALUE and (ko[7] == 0).all()
    # nothing to store
    e = torch.empty(0, H, D, dtype=torch.bfloat16, device=DEV)
    c.write(e, e, torch.empty(0, dtype=torch.int64, device=DEV))


def test_many_rows_keep_their_values():
    """A prompt's worth of tokens: what is read back equals the row to within half a step of its scale, everywhere."""
    hora = _hora()
    n, H, D, page = 20011, 4, 128, 64
    g = torch.Generator(device=DEV).manual_seed(5)
    k = torch.randn(n, H, D, device=DEV, generator=g).to(torch.bfloat16)
    v = torch.randn(n, H, D, device=DEV, generator=g).to(torch.bfloat16)
    n_pages = n // page + 2
    c = hora.PagedCache.empty(n_pages, page, H, D, F8)
    s = torch.randperm(n_pages * page, device=DEV, generator=g)[:n]
    c.write(k, v, s)
    ko, vo = (torch.empty(n, H, D, device=DEV) for _ in range(2))
    c.read(s, ko, vo)
    for x, y in ((k, ko), (v, vo)):
        x = x.float()
        unit = torch.exp2(torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448.0)))
        step = torch.maximum(x.abs() / 16.0, unit * 2.0 ** -10)     # 4-bit significands: at most 1/16 of the value; subnormal step 2^-9
        assert ((x - y).abs() <= step).all()
