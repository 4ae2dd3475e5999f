"""The example of a training step runs, and its gradients are those of the same model in 64 bits."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def exact_gradients(model, b):
    """By automatic differentiation of dense attention, from the parameters as they are."""
    p = {n: x.detach().double().requires_grad_() for n, x in model.named_parameters()}
    Hq, Hkv, D, g = model.Hq, model.Hkv, model.D, model.Hq // model.Hkv
    T = b["tokens"].numel()
    x = p["embed"][b["tokens"]]
    y = (x @ p["qkv"]).unflatten(-1, (Hq + 2 * Hkv, D))
    angle = (b["positions"].double()[:, None] * model.inv_freq)[:, None]
    c, s = torch.cos(angle), torch.sin(angle)

    def turn(z, w):
        z = z * torch.rsqrt((z * z).mean(-1, keepdim=True) + 1e-6) * w
        e, f = z[..., :D // 2], z[..., D // 2:]
        return torch.cat([e * c - f * s, e * s + f * c], -1)

    q, k, v = turn(y[:, :Hq], p["q_weight"]), turn(y[:, Hq:Hq + Hkv], p["k_weight"]).repeat_interleave(g, 1), y[:, Hq + Hkv:].repeat_interleave(g, 1)
    at = torch.arange(T, device=x.device)
    sequence = torch.searchsorted(b["seq_offsets"], at, right=True) - 1
    first = b["group_offsets"] + torch.arange(b["group_offsets"].numel(), device=x.device)          # the groups' prompts, as sequences
    group = torch.searchsorted(first, sequence, right=True) - 1
    prompt = first[group]
    seen = ((sequence[:, None] == sequence) | (sequence[None, :] == prompt[:, None])) & (at[:, None] >= at)
    z = torch.einsum("thd,khd->htk", q, k) * D ** -0.5
    out = torch.einsum("htk,khd->thd", torch.softmax(z.masked_fill(~seen, float("-inf")), -1), v)
    logits = (x + out.flatten(1) @ p["proj"]) @ p["head"]
    logp = torch.log_softmax(logits, -1).gather(1, b["tokens"].roll(-1)[:, None])[:, 0]
    (-(logp * b["signal"].double()).sum()).backward()
    return {n: x.grad for n, x in p.items()}


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gradients(dtype):
    import train_groups
    got = train_groups.run(prompts=4, dtype=dtype)
    assert got["status"] == 0
    want = exact_gradients(got["model"], got["batch"])
    # some twenty roundings between the embedding and a gradient, each of at most half a step of its value, and cancellation in the sums over
    # tokens whose weights add up to zero in every group, which their terms exceed a few times
    step = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[dtype]
    for name, x in got["model"].named_parameters():
        rel = float((x.grad.double() - want[name]).norm() / want[name].norm())
        assert rel <= 20 * step, (name, rel)


def test_the_example_as_a_program():
    done = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "train_groups.py"), "--prompts", "3"], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
    assert "status 0" in done.stdout
