"""What the tests of bad offsets and of refusals could not have noticed: writes around the buffers, and each refusal for its own reason on tensors
that are on the device; and rollouts of some thousands of tokens behind a prompt."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import test_gpu_packed_attention as tpa  # noqa: E402
from test_gpu_train_step_overlap import PATTERN, gigabytes_are_given_back, guarded, surroundings_intact  # noqa: E402, F401

DEV, BF, HF = "cuda", torch.bfloat16, torch.float16
T2 = 2000


@pytest.mark.parametrize("T,off,groups", [
    (100, [0, 40, 20, 100], None), (100, [0, 40, 400], None), (100, [-3, 40, 100], None), (100, [0, 100, 0, 100, 0, 100, 0, 100], None),
    (100, [0, 40, 60, 100], [0, 1]), (100, [0, 40, 60, 100], [0, 5]), (100, [0, 40, 60, 100], [1, 2]), (100, [0, 40, 60, 100], [0, 2, 1]), (100, [0, 40, 60, 100], [0, -1, 2]),
    (100, [1 << 62, -(1 << 62), 1 << 40], None), (100, [0, 40, 60, 100], [-(1 << 62), 1 << 62]),
    (T2, [0, T2] * 40, None), (T2, [0, T2, 0, 700, 0, T2, 0, T2, 100, T2], None),
])
@pytest.mark.parametrize("causal", [True, False])
def test_bad_offsets_touch_nothing_else(T, off, groups, causal):
    from paper_2605_07114_b200 import hora
    Hq, Hkv, D = 8, 2, 64
    q, k, v, dout = tpa.inputs(T, Hq, Hkv, D, BF, 27)
    i64 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int64, device=DEV)  # noqa: E731
    off, groups, status = i64(off), i64(groups), torch.zeros(1, dtype=torch.int32, device=DEV)
    S = off.numel() - 1
    made = {n: guarded(T * h * D * 2) for n, h in (("out", Hq), ("dq", Hq), ("dk", Hkv), ("dv", Hkv))}
    rows = {n: x[0].view(BF).view(T, -1, D) for n, x in made.items()}
    made["lse"] = guarded(T * Hq * 4)
    lse = made["lse"][0].view(torch.float32).view(T, Hq)
    made["forward"], made["backward"] = (guarded(hora.hora_packed_attention_workspace_bytes(T, S, Hq, Hkv, D, b)) for b in (False, True))
    hora.hora_packed_attention(q, k, v, off, groups, D ** -0.5, causal, rows["out"], lse, made["forward"][0], status)
    torch.cuda.synchronize()
    assert int(status) == 2
    status.zero_()
    hora.hora_packed_attention_backward(q, k, v, rows["out"], lse, dout, off, groups, D ** -0.5, causal, rows["dq"], rows["dk"], rows["dv"], made["backward"][0], status)
    torch.cuda.synchronize()
    assert int(status) == 2
    for name, (_, around) in made.items():
        assert surroundings_intact(around), name


def test_tokens_of_no_sequence_and_what_lies_around():
    """Good offsets: exactly the rows of sequences are written."""
    from paper_2605_07114_b200 import hora
    T, off, Hq, Hkv, D = 333, [30, 30, 131, 300], 4, 1, 128
    q, k, v, dout = tpa.inputs(T, Hq, Hkv, D, HF, 28)
    o = torch.tensor(off, device=DEV)
    made = {n: guarded(T * h * D * 2) for n, h in (("out", Hq), ("dq", Hq), ("dk", Hkv), ("dv", Hkv))}
    rows = {n: x[0].view(HF).view(T, -1, D) for n, x in made.items()}
    lse_bytes, lse_around = guarded(T * Hq * 4)
    lse = lse_bytes.view(torch.float32).view(T, Hq)
    for backward in (False, True):
        ws, ws_around = guarded(hora.hora_packed_attention_workspace_bytes(T, 3, Hq, Hkv, D, backward))
        if backward:
            hora.hora_packed_attention_backward(q, k, v, rows["out"], lse, dout, o, None, 0.1, True, rows["dq"], rows["dk"], rows["dv"], ws)
        else:
            hora.hora_packed_attention(q, k, v, o, None, 0.1, True, rows["out"], lse, ws)
        torch.cuda.synchronize()
        assert surroundings_intact(ws_around)
    tpa_rows = {"out": rows["out"], "lse": lse, "dq": rows["dq"], "dk": rows["dk"], "dv": rows["dv"]}
    assert surroundings_intact(lse_around) and all(surroundings_intact(a) for _, a in made.values())
    for name, x in tpa_rows.items():
        flat = x.reshape(T, -1).view(torch.uint8)
        assert bool((flat[:off[0]] == PATTERN).all()) and bool((flat[off[-1]:] == PATTERN).all()), name
        assert bool((flat[off[0]:off[-1]] != PATTERN).any(1).all()), name


def cuda(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype, device=DEV)


def test_each_refusal_of_the_rotation_for_its_own_reason():
    from paper_2605_07114_b200 import hora
    q, k, pos, f = cuda(10, 4, 64), cuda(10, 2, 64), cuda(10, dtype=torch.int32), cuda(32, dtype=torch.float64)
    good = dict(q=q, k=k, positions=pos, inv_freq=f, q_out=cuda(10, 4, 64), k_out=cuda(10, 2, 64))
    hora.hora_qk_rotate(**good)
    for over, reason in (
        (dict(k=k.float()), "of one type"), (dict(k=k[:5]), "of one type"), (dict(q=None, k=None, q_out=None, k_out=None), "or one of them"), (dict(q=q[0]), "q.*n, Hq, D"),
        (dict(q_out=q[:, :2]), "q_out must be"), (dict(q_out=q.float()), "q_out must be"), (dict(q_out=None), "q_out is missing"), (dict(k=None), "k_out is given without"),
        (dict(k_out=cuda(10, 64, 2).transpose(1, 2)), "k_out.*next to each other"), (dict(positions=pos.long()), "positions must be"), (dict(positions=pos[:9]), "one value for each token"),
        (dict(positions=None), "one value for each token"), (dict(inv_freq=f.float()), "inv_freq must be"), (dict(inv_freq=f[None]), "inv_freq must have one"),
        (dict(q_weight=cuda(64)), "q_weight must be"), (dict(k_weight=cuda(63, dtype=torch.float32)), "k_weight must hold 64"),
        (dict(positions=pos.cpu()), "positions must be a contiguous CUDA"), (dict(q=q.cpu()), "q must be a CUDA"),
    ):
        with pytest.raises(ValueError, match=reason):
            hora.hora_qk_rotate(**{**good, **over})


def test_each_refusal_of_the_attention_for_its_own_reason():
    from paper_2605_07114_b200 import hora
    q, k, off = cuda(10, 4, 64), cuda(10, 2, 64), torch.tensor([0, 4, 10], device=DEV)
    ws = torch.zeros(1 << 26, dtype=torch.uint8, device=DEV)
    good = dict(q=q, k=k, v=k.clone(), seq_offsets=off, group_offsets=None, sm_scale=0.1, causal=True, out=cuda(10, 4, 64), lse=cuda(10, 4, dtype=torch.float32), workspace=ws)
    back = {**good, "dout": q, "dq": cuda(10, 4, 64), "dk": cuda(10, 2, 64), "dv": cuda(10, 2, 64)}
    hora.hora_packed_attention(**good)
    hora.hora_packed_attention_backward(**back)
    both = [
        (dict(v=k.float()), "v must be"), (dict(k=k.float()), "k must be"), (dict(v=k[:, :1]), "v must be"), (dict(v=k[:9]), "v must be"), (dict(q=q[0]), "q must have the shape"),
        (dict(q=cuda(10, 64, 4).transpose(1, 2)), "q.*next to each other"), (dict(seq_offsets=off.int()), "seq_offsets must be"), (dict(seq_offsets=off[None]), "seq_offsets must have one"),
        (dict(seq_offsets=off[:0]), "seq_offsets must have one"), (dict(group_offsets=off[None]), "group_offsets must have one"), (dict(out=q[:, :2]), "out must be"),
        (dict(out=q.float()), "out must be"), (dict(lse=cuda(10, 3, dtype=torch.float32)), "lse must hold 40"), (dict(lse=cuda(10, 4)), "lse must be"),
        (dict(workspace=ws.int()), "workspace must be"), (dict(status_dev=off), "status_dev must be"), (dict(v=k.cpu()), "v must be a CUDA"), (dict(seq_offsets=off.cpu()), "seq_offsets must be"),
    ]
    for call, args, cases in ((hora.hora_packed_attention, good, both), (hora.hora_packed_attention_backward, back, both + [
        (dict(lse=None), "lse is missing"), (dict(dout=q.float()), "dout must be"), (dict(dout=q[:, :3]), "dout must be"), (dict(dq=k), "dq must be"), (dict(dk=q), "dk must be"),
        (dict(dv=k.float()), "dv must be"), (dict(dout=q[:, :1].expand(10, 4, 64)), "dout.*next to each other"),
    ])):
        for over, reason in cases:
            with pytest.raises(ValueError, match=reason):
                call(**{**args, **over})
        with pytest.raises(hora.HoraError) as e:
            call(**{**args, "workspace": ws[:256]})
        assert e.value.code == hora.ERR_WORKSPACE
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
def test_long_rollouts_of_a_group(dtype, D):
    groups = [[300, 4500, 2100, 1, 3700], [1025, 2047]]
    off, first = tpa.offsets([n for g in groups for n in g]), tpa.offsets([len(g) - 1 for g in groups])
    x = tpa.inputs(off[-1], 4, 2, D, dtype, 29)
    got, status = tpa.run(*x, off, first)
    assert status == 0
    tpa.check(got, *x, off, first)
