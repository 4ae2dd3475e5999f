"""One policy-gradient step over rollout groups, from the allocation to the gradients.

``hora_allocate`` says how many rollouts each prompt gets; the rollouts (made up here) lie packed behind their prompts, each prompt once;
a stand-in for a language model (one attention layer with random weights over a small vocabulary) scores them with every rollout
attending to its group's prompt, and the advantages weigh the tokens.  ``rotate`` and ``attend`` make the library's calls
differentiable for torch.

    python examples/train_groups.py [--prompts 6] [--dtype bf16]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2605_07114_b200 import hora  # noqa: E402

DEV = "cuda"


class rotate(torch.autograd.Function):
    """Norm and rotation of queries and keys; the gradients of the head weights come with it."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, inv_freq):
        op = hora.QkRotation(inv_freq, q.shape[2], q_weight=q_weight, k_weight=k_weight)
        ctx.op, ctx.positions = op, positions
        ctx.save_for_backward(q, k)
        return op.run(q, k, positions)

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        q, k = ctx.saved_tensors
        dwq, dwk = (torch.empty(q.shape[2], device=q.device) for _ in range(2))
        dq, dk = ctx.op.backward(dq_out.contiguous(), dk_out.contiguous(), q, k, ctx.positions, dq_weight=dwq, dk_weight=dwk)
        return dq, dk, dwq, dwk, None, None


class attend(torch.autograd.Function):
    """Attention of the packed tokens, a group's prompt shared by its rollouts.  Workspaces live for a call; an object that owns the output must not be kept
    for the backward pass: output, graph and object would hold each other, and their memory."""

    @staticmethod
    def forward(ctx, q, k, v, seq_offsets, group_offsets, status):
        out, lse = torch.empty(q.shape, dtype=q.dtype, device=q.device), torch.empty(q.shape[:2], device=q.device)
        ctx.at = seq_offsets, group_offsets, q.shape[2] ** -0.5, True
        ctx.status = status
        hora.hora_packed_attention(q, k, v, *ctx.at, out, lse, attend.workspace(q, k, seq_offsets, False), status)
        ctx.save_for_backward(q, k, v, out, lse)
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse = ctx.saved_tensors
        grads = [torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v)]
        hora.hora_packed_attention_backward(q, k, v, out, lse, dout.contiguous(), *ctx.at, *grads, attend.workspace(q, k, ctx.at[0], True), ctx.status)
        return (*grads, None, None, None)

    @staticmethod
    def workspace(q, k, seq_offsets, backward):
        T, Hq, D = q.shape
        need = hora.hora_packed_attention_workspace_bytes(T, seq_offsets.numel() - 1, Hq, k.shape[1], D, backward)
        return torch.empty(need, dtype=torch.uint8, device=q.device)


class Model(torch.nn.Module):
    def __init__(self, V=211, Hq=6, Hkv=2, D=64, dtype=torch.bfloat16, seed=0):
        super().__init__()
        g = torch.Generator(device=DEV).manual_seed(seed)
        E = Hq * D
        w = lambda *s: torch.nn.Parameter((torch.randn(*s, device=DEV, generator=g) * s[0] ** -0.5).to(dtype))  # noqa: E731
        self.Hq, self.Hkv, self.D = Hq, Hkv, D
        self.embed, self.qkv, self.proj, self.head = w(V, E), w(E, (Hq + 2 * Hkv) * D), w(E, E), w(E, V)
        self.embed.data *= V ** 0.5
        self.q_weight, self.k_weight = (torch.nn.Parameter(torch.ones(D, device=DEV)) for _ in range(2))
        self.inv_freq = 10000.0 ** (-torch.arange(0, D, 2, device=DEV, dtype=torch.float64) / D)

    def forward(self, tokens, positions, seq_offsets, group_offsets, status):
        x = self.embed[tokens]
        y = (x @ self.qkv).unflatten(-1, (self.Hq + 2 * self.Hkv, self.D))
        q, k, v = y.split([self.Hq, self.Hkv, self.Hkv], 1)
        q, k = rotate.apply(q, k, self.q_weight, self.k_weight, positions, self.inv_freq)
        out = attend.apply(q, k, v, seq_offsets, group_offsets, status)
        return (x + out.flatten(1) @ self.proj) @ self.head


def batch(prompts, seed=0):
    """The allocation and made-up rollouts: tokens packed group by group, the group's prompt and then its rollouts."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    N, B, G0 = prompts, 6 * prompts, 2
    c = torch.randint(0, G0 + 1, (N,), device=DEV, generator=g, dtype=torch.int32)
    cap = torch.full((N,), 16, dtype=torch.int32, device=DEV)
    alloc = hora.Allocator(N, 16, G0, exact_int=True, materialise=False, shared_int_prior=True)
    _, _, group_offsets = alloc.run(None, None, 1.0, 1.0, c, cap, 0, B)
    R = N * G0 + B
    group = torch.searchsorted(group_offsets, torch.arange(R, device=DEV), right=True) - 1
    lengths = torch.randint(20, 90, (N + R,), device=DEV, generator=g)             # of the prompts and rollouts, in the packed order
    seq_offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lengths.cumsum(0)])
    T = int(seq_offsets[-1])
    sequence = torch.repeat_interleave(torch.arange(N + R, device=DEV), lengths)
    is_prompt = torch.zeros(N + R, dtype=torch.bool, device=DEV)
    is_prompt[group_offsets[:-1] + torch.arange(N, device=DEV)] = True
    prompt_len = lengths[is_prompt]
    starts_at = torch.zeros(N + R, dtype=torch.int64, device=DEV)                  # a rollout goes on where its prompt ends
    starts_at[~is_prompt] = prompt_len[group]
    positions = (torch.arange(T, device=DEV) - seq_offsets[sequence] + starts_at[sequence]).to(torch.int32)
    tokens = torch.randint(0, 211, (T,), device=DEV, generator=g)
    # rewards -> advantages and weights of the rollouts' tokens, zeros for the prompts'
    rewards = torch.randint(0, 2, (R,), device=DEV, generator=g).float()
    own = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lengths[~is_prompt].cumsum(0)])
    adv, weight = (torch.empty(int(own[-1]), device=DEV) for _ in range(2))
    hora.hora_group_advantage_tokens(rewards, group_offsets, N, own, R, int(own[-1]), hora.ADV_GRPO, 1e-6, 0, adv, weight)
    signal = torch.zeros(T, device=DEV)
    signal[~is_prompt[sequence]] = adv * weight
    signal[seq_offsets[1:] - 1] = 0                                                # the last token of a sequence has no next one
    return dict(tokens=tokens, positions=positions, seq_offsets=seq_offsets, group_offsets=group_offsets, signal=signal)


def run(prompts=6, dtype="bf16", seed=0):
    model = Model(dtype={"bf16": torch.bfloat16, "fp16": torch.float16}[dtype], seed=seed)
    b = batch(prompts, seed)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    logits = model(b["tokens"], b["positions"], b["seq_offsets"], b["group_offsets"], status)
    logp = torch.log_softmax(logits.float(), -1).gather(1, b["tokens"].roll(-1)[:, None])[:, 0]
    loss = -(logp * b["signal"]).sum()
    loss.backward()
    torch.cuda.synchronize()
    return dict(model=model, batch=b, loss=float(loss.detach()), status=int(status))


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--prompts", type=int, default=6)
    ap.add_argument("--dtype", choices=("bf16", "fp16"), default="bf16")
    a = ap.parse_args()
    got = run(a.prompts, a.dtype)
    n = sum(p.grad.float().norm().item() ** 2 for p in got["model"].parameters()) ** 0.5
    print(f"{got['batch']['tokens'].numel()} tokens of {a.prompts} groups: loss {got['loss']:.5f}, norm of the gradient {n:.5f}, status {got['status']}")
