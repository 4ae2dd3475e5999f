"""What the calls for prompts and training steps refuse from their arguments alone, before the device is touched (no GPU needed), and
that calls with nothing to do succeed."""
from __future__ import annotations

import pytest

OK, INVALID, WORKSPACE = 0, 1, 6
F32, BF16, F16, E4M3 = range(4)
P = 0x10000          # an aligned address that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    from paper_2605_07114_b200 import build, hora
    build.build()
    return hora.load()


def rotate(lib, **over):
    a = dict(q=P, k=P, dt=BF16, qs=1024, ks=256, n=5, Hq=8, Hk=2, D=128, pos=P, f=P, rot=128, layout=0, wq=P, wk=P, eps=1e-6, qo=P, ko=P, qos=1024, kos=256)
    a.update(over)
    return lib.hora_qk_rotate(a["q"], a["k"], a["dt"], a["qs"], a["ks"], a["n"], a["Hq"], a["Hk"], a["D"], a["pos"], a["f"], a["rot"], a["layout"], a["wq"], a["wk"],
                              a["eps"], a["qo"], a["ko"], a["qos"], a["kos"], None)


ROTATE_BAD = [dict(n=-1), dict(n=1 << 31), dict(Hq=-1), dict(Hk=-1), dict(Hq=0, Hk=0), dict(Hq=1 << 17), dict(D=96), dict(D=256), dict(rot=-16), dict(rot=8), dict(rot=144),
              dict(layout=2), dict(layout=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(dt=E4M3), dict(dt=9)]


@pytest.mark.parametrize("over", ROTATE_BAD + [
    dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(q=P + 8), dict(k=P + 2), dict(qo=P + 4), dict(ko=P + 8), dict(qs=1023), dict(qs=1028), dict(ks=248),
    dict(qos=1020), dict(kos=260), dict(pos=None), dict(f=None), dict(f=P + 4), dict(pos=P + 2), dict(wq=P + 1), dict(wk=P + 2),
])
def test_rotate(lib, over):
    assert rotate(lib, **over) == INVALID


def test_rotate_without_tokens(lib):
    assert rotate(lib, n=0, q=None, k=None, qo=None, ko=None, pos=None, f=None) == OK


def rotate_backward(lib, **over):
    a = dict(gq=P, gk=P, dt=BF16, gqs=1024, gks=256, q=P, k=P, qs=1024, ks=256, n=5, Hq=8, Hk=2, D=128, pos=P, f=P, rot=128, layout=0, wq=P, wk=P, eps=1e-6, dq=P, dk=P,
             dqs=1024, dks=256, dwq=P, dwk=P, ws=P, wb=1 << 30)
    a.update(over)
    return lib.hora_qk_rotate_backward(a["gq"], a["gk"], a["dt"], a["gqs"], a["gks"], a["q"], a["k"], a["qs"], a["ks"], a["n"], a["Hq"], a["Hk"], a["D"], a["pos"], a["f"],
                                       a["rot"], a["layout"], a["wq"], a["wk"], a["eps"], a["dq"], a["dk"], a["dqs"], a["dks"], a["dwq"], a["dwk"], a["ws"], a["wb"], None)


@pytest.mark.parametrize("over", ROTATE_BAD + [
    dict(gq=None), dict(gk=None), dict(dq=None), dict(dk=None), dict(q=None), dict(k=None), dict(gq=P + 8), dict(dk=P + 2), dict(q=P + 4), dict(gqs=1016), dict(dks=252),
    dict(qs=1030), dict(pos=None), dict(f=None), dict(wq=None), dict(wk=None), dict(f=P + 4), dict(dwq=P + 2), dict(dwk=P + 1),
])
def test_rotate_backward(lib, over):
    assert rotate_backward(lib, **over) == INVALID


def test_rotate_backward_workspace(lib):
    need = lib.hora_qk_rotate_backward_workspace_bytes(128)
    assert need >= 2 * 128 * 4 and lib.hora_qk_rotate_backward_workspace_bytes(64) * 2 == need and lib.hora_qk_rotate_backward_workspace_bytes(96) == 0
    assert rotate_backward(lib, ws=None) == WORKSPACE and rotate_backward(lib, ws=P + 16) == WORKSPACE and rotate_backward(lib, wb=need - 1) == WORKSPACE
    assert rotate_backward(lib, n=0, dwq=None, dwk=None, gq=None, ws=None) == OK


COMMON = dict(q=P, k=P, v=P, dt=BF16, qs=1024, ks=256, vs=512, T=100, so=P, S=4, go=P, N=2, Hq=8, Hkv=2, D=128, scale=0.1, causal=1, out=P, os=1024, lse=P, ws=P, wb=1 << 40)


def attention(lib, **over):
    a = dict(COMMON, **over)
    return lib.hora_packed_attention(a["q"], a["k"], a["v"], a["dt"], a["qs"], a["ks"], a["vs"], a["T"], a["so"], a["S"], a["go"], a["N"], a["Hq"], a["Hkv"], a["D"], a["scale"],
                                     a["causal"], a["out"], a["os"], a["lse"], None, a["ws"], a["wb"], None)


def attention_backward(lib, **over):
    a = dict(COMMON, do=P, dos=1024, dq=P, dk=P, dv=P, dqs=1024, dks=256, dvs=264)
    a.update(over)
    return lib.hora_packed_attention_backward(a["q"], a["k"], a["v"], a["out"], a["lse"], a["do"], a["dt"], a["qs"], a["ks"], a["vs"], a["os"], a["dos"], a["T"], a["so"], a["S"], a["go"],
                                              a["N"], a["Hq"], a["Hkv"], a["D"], a["scale"], a["causal"], a["dq"], a["dk"], a["dv"], a["dqs"], a["dks"], a["dvs"], None, a["ws"], a["wb"], None)


ATTENTION_BAD = [
    dict(T=-1), dict(T=1 << 31), dict(S=-1), dict(S=1 << 30), dict(N=-1), dict(N=5), dict(N=0), dict(go=None), dict(Hq=0), dict(Hkv=0), dict(Hq=7), dict(Hq=1 << 17), dict(D=96),
    dict(D=256), dict(dt=F32), dict(dt=E4M3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(causal=2), dict(causal=-1),
    dict(q=None), dict(k=None), dict(v=None), dict(so=None), dict(out=None), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(out=P + 8), dict(qs=1023), dict(qs=1028), dict(ks=248), dict(vs=252),
    dict(os=1020), dict(os=1000), dict(so=P + 4), dict(go=P + 2), dict(lse=P + 2),
]


@pytest.mark.parametrize("over", ATTENTION_BAD)
def test_attention(lib, over):
    assert attention(lib, **over) == INVALID


@pytest.mark.parametrize("over", ATTENTION_BAD + [
    dict(lse=None), dict(do=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(do=P + 8), dict(dq=P + 4), dict(dk=P + 2), dict(dv=P + 8), dict(dos=1016), dict(dqs=1023), dict(dks=255), dict(dvs=248),
])
def test_attention_backward(lib, over):
    assert attention_backward(lib, **over) == INVALID


def test_attention_workspace(lib):
    forward, backward = (lib.hora_packed_attention_workspace_bytes(100, 4, 8, 2, 128, b) for b in (0, 1))
    assert forward % 256 == 0 and backward % 256 == 0 and backward > forward > 0
    for call, need in ((attention, forward), (attention_backward, backward)):
        assert call(lib, ws=None) == WORKSPACE and call(lib, ws=P + 16) == WORKSPACE and call(lib, wb=need - 1) == WORKSPACE
        assert call(lib, T=0, q=None) == OK and call(lib, S=0, N=0, go=None, so=None) == OK
    for bad in ((-1, 4, 8, 2, 128), (100, -1, 8, 2, 128), (100, 4, 8, 3, 128), (100, 4, 8, 2, 96), (100, 4, 0, 2, 128)):
        assert lib.hora_packed_attention_workspace_bytes(*bad, 0) == 0


def test_the_binding_checks_shapes_types_and_devices():
    torch = pytest.importorskip("torch")
    from paper_2605_07114_b200 import hora
    bf = torch.bfloat16
    q, k = torch.zeros(10, 4, 64, dtype=bf), torch.zeros(10, 2, 64, dtype=bf)
    pos, f = torch.zeros(10, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    for args in ((q, k.float(), pos, f, q, k), (q, k[:5], pos, f, q, k), (q, k, pos, f, q[:, :2], k), (None, None, pos, f, None, None), (q, None, pos, f, q, k),
                 (q, k, pos, f, q, k)):                                            # the last: not on a device
        with pytest.raises(ValueError):
            hora.hora_qk_rotate(*args)
    off, ws, lse = torch.zeros(3, dtype=torch.int64), torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(10, 4)
    for args in ((q, k, k, off, None, 0.1, True, q, lse, ws), (q, k, k.float(), off, None, 0.1, True, q, lse, ws), (q, k, k[:, :1], off, None, 0.1, True, q, lse, ws),
                 (q[0], k, k, off, None, 0.1, True, q, lse, ws)):
        with pytest.raises(ValueError):
            hora.hora_packed_attention(*args)
    with pytest.raises(ValueError):
        hora.PackedAttention(off, 10, 4, 3, 64, bf)                                # four heads over three
    with pytest.raises(ValueError):
        hora.PackedAttention(off, 10, 4, 2, 64, torch.float32)
    with pytest.raises(ValueError):
        hora.PackedAttention(off[:0], 10, 4, 2, 64, bf)
    with pytest.raises(ValueError):
        hora.QkRotation(None, 64)
