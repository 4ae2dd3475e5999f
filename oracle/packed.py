"""The operators of prompts and training steps, in 64 bits and one sequence after the other, with bounds on what a computation that
rounds as the library says it does may be off by.  torch tensors of any device; shares no code with the library."""
from __future__ import annotations

import math

import torch


def sequences(seq_offsets, group_offsets=None):
    """(token range, prompt's token range or None) of every sequence."""
    ranges = list(zip(seq_offsets[:-1], seq_offsets[1:]))
    prompt = [None] * len(ranges)
    if group_offsets is not None:
        for i in range(len(group_offsets) - 1):
            for r in range(group_offsets[i], group_offsets[i + 1]):
                prompt[r + i + 1] = ranges[group_offsets[i] + i]
    return list(zip(ranges, prompt))


def packed_attention(q, k, v, seq_offsets, group_offsets=None, causal=True, scale=None, dout=None, step=None, tiny=0.0):
    """out, lse (and dq, dk, dv where dout is given), with bounds out_tol .. for elements computed by products in 32 bits whose weights are
    rounded to a type of the half step `step` relative to the value, and of `tiny` for the smallest of them; results are rounded so too."""
    T, Hq, D = q.shape
    g, scale = Hq // k.shape[1], D ** -0.5 if scale is None else scale
    q, k, v = q.double(), k.double(), v.double()
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    like = lambda: torch.zeros_like(q)  # noqa: E731
    r = {"out": like(), "lse": torch.full((T, Hq), -math.inf, dtype=torch.float64, device=q.device)}
    tol = {"out": like(), "lse": torch.zeros_like(r["lse"])}
    if dout is not None:
        dout = dout.double()
        for n in ("dq", "dk", "dv"):
            r[n], tol[n] = like(), like()
    u = 0.0 if step is None else step
    seqs = sequences(seq_offsets, group_offsets)
    # fp16 holds gradients of scores relative to a power of two that follows from the largest rows
    largest = 0.0
    if dout is not None and seq_offsets[-1] > seq_offsets[0]:
        mine = slice(seq_offsets[0], seq_offsets[-1])
        largest = 2.0 * float(dout[mine].norm(dim=-1).max()) * float(v[mine].norm(dim=-1).max())
    for (a, b), shared in seqs:
        if a == b:
            continue
        at = torch.arange(a, b, device=q.device)
        if shared is not None:
            at = torch.cat([torch.arange(*shared, device=q.device), at])
        Q, K, V = (x.transpose(0, 1) for x in (q[a:b], k[at], v[at]))                 # [H, rows, D], [H, keys, D]
        s = scale * Q @ K.transpose(1, 2)
        if causal:
            s = s.masked_fill(at[None, :] > torch.arange(a, b, device=q.device)[:, None], -math.inf)
        lse = torch.logsumexp(s, -1, keepdim=True)
        P = torch.exp(s - lse)
        o = P @ V
        # scores: D products added in 32 bits, then a difference and an exponential of them
        e_s = scale * (D + 2) * 2.0 ** -24 * (Q.abs() @ K.abs().transpose(1, 2)) + 2.0 ** -22 * (1 + s.abs().clamp(max=1e9).nan_to_num(0.0) + lse.abs())
        e_s = torch.where(P > 0, e_s, torch.zeros_like(e_s))
        e_row = (P * e_s).sum(-1, keepdim=True) + at.numel() * 2.0 ** -24
        eP = P * (e_s + e_row + u) + tiny
        eP = torch.where(torch.isinf(s), torch.zeros_like(eP), eP)
        e_o = eP @ V.abs() + u * o.abs() + (at.numel() + 4) * 2.0 ** -24 * (P @ V.abs())
        r["out"][a:b], tol["out"][a:b] = o.transpose(0, 1), e_o.transpose(0, 1)
        r["lse"][a:b], tol["lse"][a:b] = lse[..., 0].T, (e_row + 2.0 ** -22 * (1 + lse.abs()))[..., 0].T
        if dout is None:
            continue
        dO = dout[a:b].transpose(0, 1)
        dP, delta = dO @ V.transpose(1, 2), (dO * o).sum(-1, keepdim=True)
        dS = P * (dP - delta)
        # weights come from lse here, delta from the rounded output
        e_w = torch.where(torch.isinf(s), torch.zeros_like(P), P * (e_s + e_row + 2.0 ** -21))
        e_delta = (dO.abs() * e_o).sum(-1, keepdim=True) + D * 2.0 ** -23 * (dO * o).abs().sum(-1, keepdim=True)
        e_dP = D * 2.0 ** -23 * (dO.abs() @ V.abs().transpose(1, 2)) + e_delta
        e_dS = u * dS.abs() + P * e_dP + e_w * (dP - delta).abs()
        e_dS = torch.where(torch.isinf(s), torch.zeros_like(P), e_dS + (tiny * 2.0 ** -14 * largest))
        eP = torch.where(torch.isinf(s), torch.zeros_like(P), e_w + u * P + tiny * 2.0 ** -10)
        more = 1 + 2.0 ** -10                        # sums in 32 bits of thousands of terms, next to what their terms are off by
        r["dq"][a:b] = scale * (dS @ K).transpose(0, 1)
        tol["dq"][a:b] = more * scale * ((e_dS + 2.0 ** -20 * dS.abs()) @ K.abs()).transpose(0, 1)
        r["dk"].index_add_(0, at, scale * (dS.transpose(1, 2) @ Q).transpose(0, 1))
        tol["dk"].index_add_(0, at, more * scale * ((e_dS + 2.0 ** -20 * dS.abs()).transpose(1, 2) @ Q.abs()).transpose(0, 1))
        r["dv"].index_add_(0, at, (P.transpose(1, 2) @ dO).transpose(0, 1))
        tol["dv"].index_add_(0, at, more * ((eP + 2.0 ** -20 * P).transpose(1, 2) @ dO.abs()).transpose(0, 1))
    if dout is not None:
        for n in ("dk", "dv"):                       # a head's gradient is the sum over the query heads that read it
            r[n], tol[n] = (x.reshape(T, Hq // g, g, D).sum(2) for x in (r[n], tol[n]))
        for n in ("dq", "dk", "dv"):
            tol[n] = tol[n] * (1 + u) + u * r[n].abs() + tiny
    tol["out"] = tol["out"] * (1 + u) + tiny
    return r, tol


def qk_rotate(x, positions, inv_freq, pairs, w=None, eps=0.0, dy=None):
    """y (and dx, dw) of rows x [n, H, D], from the formulas."""
    x, rot = x.double(), 2 * len(inv_freq)
    angle = (positions.double()[:, None] * inv_freq.double())[:, None, :]
    c, s = torch.cos(angle), torch.sin(angle)

    def turn(z, s):
        y = z.clone()
        a, b = (z[..., 0:rot:2], z[..., 1:rot:2]) if pairs else (z[..., :rot // 2], z[..., rot // 2:rot])
        first, second = a * c - b * s, a * s + b * c
        if pairs:
            y[..., 0:rot:2], y[..., 1:rot:2] = first, second
        else:
            y[..., :rot // 2], y[..., rot // 2:rot] = first, second
        return y

    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) if w is not None else torch.ones_like(x[..., :1])
    z = x * r * w.double() if w is not None else x
    y = turn(z, s)
    if dy is None:
        return y
    g = turn(dy.double(), -s)
    if w is None:
        return y, g, None
    u = x * r
    wg = w.double() * g
    return y, r * (wg - u * (u * wg).mean(-1, keepdim=True)), (u * g).sum((0, 1))
