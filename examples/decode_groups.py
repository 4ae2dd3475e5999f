"""Rollout groups from the allocation to the advantages, with the library's operators in between.

A stand-in for a language model (one attention layer with random weights over a small vocabulary) generates the rollouts
that ``hora_allocate`` hands out: every group shares its prompt's cache, which is quantised as it is written; each step
verifies a few drafted tokens of every rollout.  Then the rewards become advantages.

    python examples/decode_groups.py [--prompts 15] [--steps 8] [--drafts 3] [--dtype e4m3]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2605_07114_b200 import hora  # noqa: E402

DEV = "cuda"


class Model:
    """Token embedding, one attention layer, output projection.  Positions enter by an additive code."""

    def __init__(self, V=997, Hq=8, Hkv=2, D=64, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        E = Hq * D
        w = lambda *s: (torch.randn(*s, device=DEV, generator=g) * s[0] ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.V, self.Hq, self.Hkv, self.D, self.E = V, Hq, Hkv, D, E
        self.embed, self.qkv, self.proj, self.head = w(V, E) * V ** 0.5, w(E, (Hq + 2 * Hkv) * D), w(E, E), w(E, V) * 2.0
        self.draft_table = torch.softmax((self.embed @ self.head).float(), -1)      # a bigram model drafts

    def project(self, tokens, positions):
        """(hidden, q [.., Hq, D], k, v [.., Hkv, D]): views into one projection."""
        p = positions.unsqueeze(-1) / 10000 ** (torch.arange(self.E, device=DEV) / self.E)
        x = self.embed[tokens] + torch.sin(p).to(torch.bfloat16)
        y = x @ self.qkv
        q, k, v = y.split([self.Hq * self.D, self.Hkv * self.D, self.Hkv * self.D], -1)
        return x, q.unflatten(-1, (self.Hq, self.D)), k.unflatten(-1, (self.Hkv, self.D)), v.unflatten(-1, (self.Hkv, self.D))

    def probabilities(self, x, attended):
        return torch.softmax((x + attended.flatten(-2) @ self.proj) @ self.head, -1, dtype=torch.float32)


def run(prompts=15, steps=8, drafts=3, dtype="e4m3", seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    model, page, T, G0 = Model(), 16, drafts + 1, 8
    N, B = prompts, 24 * prompts

    # Phase A has counted c correct ones among G0 rollouts of each prompt; the rest of the budget is allocated
    c = torch.randint(0, G0 + 1, (N,), device=DEV, generator=g, dtype=torch.int32)
    cap = torch.full((N,), 64, dtype=torch.int32, device=DEV)
    alloc = hora.Allocator(N, 64, G0, exact_int=True, materialise=False, shared_int_prior=True)
    _, _, group_offsets = alloc.run(None, None, 1.0, 1.0, c, cap, 0, B)
    R = N * G0 + B

    # pages: the prompts' first, then every rollout's own
    prompt_len = torch.randint(20, 200, (N,), device=DEV, generator=g, dtype=torch.int32)
    per_prompt, per_rollout = -(-200 // page), -(-(steps * T + T) // page)
    prefix_pages = torch.arange(N * per_prompt, device=DEV, dtype=torch.int32).reshape(N, per_prompt)
    suffix_pages = (N * per_prompt + torch.arange(R * per_rollout, device=DEV, dtype=torch.int32)).reshape(R, per_rollout)
    types = {"e4m3": torch.float8_e4m3fn, "bf16": torch.bfloat16}
    cache = hora.PagedCache.empty(N * per_prompt + R * per_rollout, page, model.Hkv, model.D, types[dtype])
    status = torch.zeros(1, dtype=torch.int32, device=DEV)

    # the prompts' keys and values; slots of tokens beyond a prompt's length are negative: not stored
    at = torch.arange(200, device=DEV)
    slots = prefix_pages.long()[:, at // page] * page + at % page
    slots = torch.where(at < prompt_len[:, None], slots, -1)
    text = torch.randint(0, model.V, (N, 200), device=DEV, generator=g)
    _, _, k, v = model.project(text, at.expand(N, 200).float())
    cache.write(k.flatten(0, 1), v.flatten(0, 1), slots.flatten(), status)

    group = torch.searchsorted(group_offsets, torch.arange(R, device=DEV), right=True) - 1
    last = text.gather(1, (prompt_len.long() - 1)[:, None])[group, 0]              # the last token known of each rollout
    own_len = torch.zeros(R, dtype=torch.int32, device=DEV)
    attend = hora.GroupAttention(cache, model.Hq, T, torch.bfloat16, group_offsets=group_offsets, prefix_pages=prefix_pages, prefix_len=prompt_len,
                                 suffix_pages=suffix_pages, suffix_len=own_len, status_dev=status)
    n_accepted = torch.empty(R, dtype=torch.int32, device=DEV)
    out = torch.empty(R, T, dtype=torch.int32, device=DEV)
    texts, r = [], torch.arange(R, device=DEV)
    for _ in range(steps):
        # drafts of the bigram model, with the rows they were drawn from
        tokens, rows = [last], []
        for _ in range(drafts):
            rows.append(model.draft_table[tokens[-1]])
            tokens.append(torch.multinomial(rows[-1], 1, generator=g)[:, 0])
        tokens = torch.stack(tokens, 1)                                            # [R, T]: the last known token, then the drafts
        place = own_len.long()[:, None] + torch.arange(T, device=DEV)
        x, q, k, v = model.project(tokens, (prompt_len[group][:, None] + place).float())
        slots = suffix_pages.long()[r[:, None], place // page] * page + place % page
        cache.write(k.flatten(0, 1), v.flatten(0, 1), slots.flatten(), status)
        own_len += T                                                               # the queries are the last T of the rollout's tokens
        attended, _ = attend.run(q)
        target = model.probabilities(x, attended)
        hora.hora_verify_drafts(target, torch.stack(rows, 1) if drafts else None, tokens[:, 1:].to(torch.int32).contiguous(), None, R, drafts, model.V,
                                torch.rand(R, drafts, device=DEV, generator=g), torch.rand(R, device=DEV, generator=g), n_accepted, out, status)
        own_len += n_accepted + 1 - T                                              # refused drafts are overwritten by the next step
        last = out.long()[r, n_accepted.long()]
        texts.append(out.clone())

    # a made-up reward, and the advantages of the groups
    rewards = (torch.stack(texts).long().clamp(min=0).sum((0, 2)) % 2).float()
    adv = torch.empty(R, device=DEV)
    hora.hora_group_advantage(rewards, group_offsets, N, hora.ADV_GRPO, 1e-6, 0, adv, status)
    torch.cuda.synchronize()
    return dict(status=int(status), group_offsets=group_offsets, own_len=own_len, texts=texts, n_accepted=n_accepted, adv=adv, R=R, target=target)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--prompts", type=int, default=15)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=3)
    ap.add_argument("--dtype", choices=("e4m3", "bf16"), default="e4m3")
    a = ap.parse_args()
    got = run(a.prompts, a.steps, a.drafts, a.dtype)
    made = sum(int((t >= 0).sum()) for t in got["texts"])
    print(f"{got['R']} rollouts in {a.prompts} groups, {a.steps} steps: {made} tokens, {made / got['R'] / a.steps:.2f} a step and rollout, status {got['status']}")
