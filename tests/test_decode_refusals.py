"""What the decode-step calls refuse from their arguments alone, before the device is touched (no GPU needed), and that calls
with nothing to do succeed."""
from __future__ import annotations

import ctypes as C

import pytest

OK, INVALID, WORKSPACE = 0, 1, 6
F32, BF16, F16, E4M3 = range(4)
P = 0x10000          # an aligned address that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    from paper_2605_07114_b200 import build, hora
    build.build()
    return hora.load()


def kv(lib, which="write", **over):
    a = dict(k=P, v=P, dtype=BF16, stride=256, slots=P, n=4, H=2, D=128, kc=P, vc=P, ke=P, ve=P, cache=E4M3, n_pages=8, page=16)
    a.update(over)
    if which == "write":
        return lib.hora_kv_write(a["k"], a["v"], a["dtype"], a["stride"], a["slots"], a["n"], a["H"], a["D"], a["kc"], a["vc"], a["ke"], a["ve"],
                                 a["cache"], a["n_pages"], a["page"], None, None)
    return lib.hora_kv_read(a["kc"], a["vc"], a["ke"], a["ve"], a["cache"], a["n_pages"], a["page"], a["slots"], a["n"], a["H"], a["D"], a["k"], a["v"],
                            a["dtype"], a["stride"], None, None)


@pytest.mark.parametrize("which", ["write", "read"])
@pytest.mark.parametrize("over", [
    dict(n=-1), dict(H=0), dict(D=96), dict(D=0), dict(D=256), dict(page=8), dict(page=48), dict(page=256), dict(n_pages=0), dict(dtype=E4M3), dict(dtype=7),
    dict(cache=F32), dict(cache=9), dict(stride=255), dict(stride=260), dict(k=None), dict(v=None), dict(slots=None), dict(kc=None), dict(vc=None),
    dict(ke=None), dict(ve=None), dict(k=P + 8), dict(kc=P + 4), dict(ke=P + 2),
])
def test_cache_calls(lib, which, over):
    assert kv(lib, which, **over) == INVALID


def test_cache_calls_without_tokens(lib):
    assert kv(lib, "write", n=0, k=None, v=None, slots=None) == OK and kv(lib, "read", n=0, k=None, v=None, slots=None) == OK


def attention(lib, **over):
    a = dict(q=P, dt=BF16, qs=1024, off=P, N=3, R=9, T=2, ql=None, Hq=8, Hkv=2, D=128, scale=0.1, kc=P, vc=P, ke=None, ve=None, cache=BF16, n_pages=64, page=16,
             pp=P, pld=4, pl=P, sp=P, sld=4, sl=P, out=P, os=1024, lse=None, ws=P, wb=1 << 40)
    a.update(over)
    return lib.hora_group_attention(a["q"], a["dt"], a["qs"], a["off"], a["N"], a["R"], a["T"], a["ql"], a["Hq"], a["Hkv"], a["D"], a["scale"], a["kc"], a["vc"],
                                    a["ke"], a["ve"], a["cache"], a["n_pages"], a["page"], a["pp"], a["pld"], a["pl"], a["sp"], a["sld"], a["sl"], a["out"],
                                    a["os"], a["lse"], None, a["ws"], a["wb"], None)


@pytest.mark.parametrize("over", [
    dict(N=-1), dict(N=0), dict(R=-1), dict(T=0), dict(Hq=0), dict(Hkv=0), dict(Hq=7), dict(D=80), dict(D=256), dict(R=1 << 31), dict(R=1 << 29, T=8), dict(T=2000, Hq=32),
    dict(dt=F32), dict(dt=E4M3), dict(cache=F16), dict(cache=F32), dict(cache=E4M3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(page=24), dict(n_pages=0), dict(pld=-1), dict(sld=-1), dict(pld=1 << 28), dict(q=None), dict(out=None), dict(off=None),
    dict(pl=None), dict(sl=None), dict(pp=None), dict(sp=None), dict(kc=None), dict(q=P + 2), dict(out=P + 8), dict(qs=1023), dict(qs=1028), dict(os=1016), dict(os=1030),
])
def test_attention(lib, over):
    assert attention(lib, **over) == INVALID


def test_attention_workspace(lib):
    need = lib.hora_group_attention_workspace_bytes(3, 9, 2, 8, 2, 128)
    assert need % 256 == 0 and need > 9 * 2 * 8 * 128 * 4 * 2
    assert attention(lib, ws=None) == WORKSPACE and attention(lib, ws=P + 16) == WORKSPACE and attention(lib, wb=need - 1) == WORKSPACE
    for bad in ((-1, 9, 2, 8, 2, 128), (0, 9, 2, 8, 2, 128), (3, 9, 0, 8, 2, 128), (3, 9, 2, 8, 3, 128), (3, 9, 2, 8, 2, 96)):
        assert lib.hora_group_attention_workspace_bytes(*bad) == 0
    more = lib.hora_group_attention_workspace_bytes(3, 90, 2, 8, 2, 128)
    assert more > need
    assert attention(lib, R=0, q=None, out=None) == OK


def verify(lib, **over):
    a = dict(t=P, dt=F32, ts=100, d=P, ds=100, tok=P, ln=None, R=3, K=2, V=100, ua=P, us=P, n=P, out=P)
    a.update(over)
    return lib.hora_verify_drafts(a["t"], a["dt"], a["ts"], a["d"], a["ds"], a["tok"], a["ln"], a["R"], a["K"], a["V"], a["ua"], a["us"], a["n"], a["out"], None, None)


@pytest.mark.parametrize("over", [
    dict(R=-1), dict(R=1 << 28), dict(K=-1), dict(K=256), dict(V=0), dict(V=(1 << 22) + 1, ts=1 << 23, ds=1 << 23), dict(dt=E4M3), dict(dt=5), dict(ts=99), dict(ds=99),
    dict(t=None), dict(tok=None), dict(ua=None), dict(us=None), dict(n=None), dict(out=None), dict(t=P + 2), dict(d=P + 1),
])
def test_verify_drafts(lib, over):
    assert verify(lib, **over) == INVALID


def test_verify_drafts_without_rollouts(lib):
    assert verify(lib, R=0, t=None) == OK


def test_the_binding_checks_shapes_and_types():
    torch = pytest.importorskip("torch")
    from paper_2605_07114_b200 import hora
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        hora.PagedCache.over(k, k.float())
    with pytest.raises(ValueError):
        hora.PagedCache.over(k, torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        hora.PagedCache.over(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn))     # no scale bytes
    with pytest.raises(ValueError):
        hora.PagedCache.over(k, k)                                                     # not on a device
    t = torch.zeros(3, 3, 10)
    with pytest.raises(ValueError):
        hora.hora_verify_drafts(t, None, torch.zeros(3, 3, dtype=torch.int32), None, 3, 3, 10, t, t, t, t)
