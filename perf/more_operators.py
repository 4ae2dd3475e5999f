"""The operators of prompts and of a training step over rollout groups, as cases to be measured.

Queries and keys are normed and rotated by their positions; packed sequences of different lengths attend to
themselves and, where they are rollouts of a group, to their group's prompt, which lies once among the packed tokens; a
training step takes the gradients of both.  ``run`` makes one pass through one of these operators: in plain torch
operations where ``own`` is false, through the library where it is true.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _attention(name, N, R, prompt, rollout, Hq, Hkv, D, dtype, causal, train):
    c = dict(op="attention", N=N, R=R, prompt=prompt, rollout=rollout, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, causal=causal, train=train)
    return dict(c, name=name) if name else c


def _rotate(name, n, Hq, Hk, D, rot, dtype, pairs, norm, train):
    c = dict(op="rotate", n=n, Hq=Hq, Hk=Hk, D=D, rot=rot, dtype=dtype, pairs=pairs, norm=norm, train=train)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the prompt of a single problem, before its pre-rollouts: latency counts
        _attention("prompt one", 1, 0, 211, 0, 12, 2, 128, "bf16", True, False),
        # all prompts of a training batch in one go
        _attention("prompts 60", 60, 0, 509, 0, 28, 4, 128, "bf16", True, False),
        # one long document
        _attention("prompt long fp16", 1, 0, 16381, 0, 32, 8, 128, "f16", True, False),
        # an encoder's look at the problems (predictors of the prior read them both ways), small heads, no shared keys
        _attention("both ways D=64 fp16", 64, 0, 512, 0, 12, 12, 64, "f16", False, False),
        # log-probabilities of one shard's rollouts, scored again behind their prompts
        _attention("groups 15x32", 15, 480, 413, 509, 28, 4, 128, "bf16", True, False),
        # a training step of two small groups, smaller heads
        _attention("train small D=64", 2, 16, 211, 103, 12, 2, 64, "bf16", True, True),
        # a training step of a shard: eight groups of sixteen, responses up to 1021 tokens
        _attention("train groups 8x16", 8, 128, 413, 1021, 28, 4, 128, "bf16", True, True),
        # a training step over two long traces without groups
        _attention("train long fp16", 2, 0, 8191, 0, 16, 8, 128, "f16", True, True),
        # one decode step of a shard: one new token of each rollout
        _rotate("rotate step", 480, 28, 4, 128, 128, "bf16", False, True, False),
        # the prompts of a batch
        _rotate("rotate prompts", 131072, 16, 4, 128, 128, "bf16", False, True, False),
        # a training step's packed rollouts
        _rotate("rotate train", 50021, 28, 4, 128, 128, "bf16", False, True, True),
        # a 32-bit layer that turns neighbouring values, half of each head, a ragged number of tokens
        _rotate("rotate train f32 pairs", 20011, 12, 3, 64, 32, "f32", True, True, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        if rng.random() < 0.65:
            Hkv, D = rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 128, 128])
            Hq, dtype, train = Hkv * rng.choice([1, 1, 2, 3, 4, 5, 6, 7, 8]), rng.choice(["bf16", "bf16", "f16"]), rng.random() < 0.5
            N = _log(rng, 1, 64)
            R = N * _log(rng, 1, 32) + rng.randrange(N) if rng.random() < 0.5 else 0
            c = _attention(None, N, R, _log(rng, 8, 16384), _log(rng, 8, 2048) if R else 0, Hq, Hkv, D, dtype, R > 0 or rng.random() < 0.8, train)
            like = [x for x in listed() if x["op"] == "attention" and x["train"] == train]
        else:
            D, Hk = rng.choice([64, 128, 128]), rng.randint(1, 8)
            c = _rotate(None, _log(rng, 1, 131072), Hk * rng.randint(1, 8), Hk, D, rng.choice([D, D, D // 2]), rng.choice(["bf16", "f16", "f32"]),
                        rng.random() < 0.3, rng.random() < 0.7, rng.random() < 0.5)
            like = [x for x in listed() if x["op"] == "rotate"]
        if _cost(c) <= max(_cost(x) for x in like):
            return c


def _cost(c):
    """Roughly what a pass in its plain form moves, to keep drawn cases within the listed ones."""
    if c["op"] == "attention":
        return c["Hq"] * (c["N"] * c["prompt"] ** 2 + c["R"] * c["rollout"] * (c["prompt"] + c["rollout"])) + (c["N"] * c["prompt"] + c["R"] * c["rollout"]) * c["Hq"] * c["D"]
    return c["n"] * (c["Hq"] + c["Hk"]) * c["D"] * (BYTES[c["dtype"]] / 2) * (2 if c["train"] else 1)


# ---------------------------------------------------------------------------------------------------------------
# inputs


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = np.random.Generator(np.random.PCG64(seed))
    return (_prepare_attention if case["op"] == "attention" else _prepare_rotate)(dict(case), g, rng)


def _lengths(rng, n, lo, hi):
    """n lengths in lo .. hi, two and two of one sum and an odd one out of length hi: the tokens of a case are always as many."""
    x = rng.integers(lo, hi + 1, n // 2)
    return rng.permutation(np.concatenate([x, lo + hi - x, np.full(n % 2, hi)])).astype(np.int64)


def _prepare_attention(c, g, rng):
    N, R, Hq, Hkv, D = (c[k] for k in ("N", "R", "Hq", "Hkv", "D"))
    prompt = _lengths(rng, N, max(1, c["prompt"] // 2), c["prompt"])
    sizes = 1 + rng.multinomial(R - N, rng.dirichlet(np.full(N, 2.0))) if R else np.zeros(N, np.int64)        # uneven groups, as the allocation makes them
    rollout = _lengths(rng, R, 1, c["rollout"]) if R else np.zeros(0, np.int64)
    first = np.concatenate([[0], np.cumsum(sizes)])
    lengths = np.concatenate([np.concatenate([prompt[i:i + 1], rollout[first[i]:first[i + 1]]]) for i in range(N)])
    offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    T = int(offsets[-1])
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int64)).to(DEV)  # noqa: E731
    dt = TYPES[c["dtype"]]
    # queries, keys and values side by side, as one projection writes them; queries larger than keys: some positions matter, most do not
    qkv = torch.randn(T, Hq + 2 * Hkv, D, device=DEV, generator=g)
    qkv[:, :Hq] *= 2.0
    qkv = qkv.to(dt)
    s = dict(c, T=T, q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], offsets=t(offsets), group_offsets=t(first) if R else None,
             prompt_max=int(prompt.max()), rollout_max=int(rollout.max()) if R else 0, scale=D ** -0.5)
    if c["train"]:       # tokens weigh differently: by their advantages and their rollouts' lengths
        weight = torch.exp(torch.randn(T, 1, 1, device=DEV, generator=g))
        s["dout"] = (torch.randn(T, Hq, D, device=DEV, generator=g) * weight).to(dt)
    return s


def _prepare_rotate(c, g, rng):
    n, Hq, Hk, D = (c[k] for k in ("n", "Hq", "Hk", "D"))
    dt = TYPES[c["dtype"]]
    qkv = torch.randn(n, Hq + 2 * Hk, D, device=DEV, generator=g).to(dt)           # a fused projection; the values stay as they are
    s = dict(c, q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hk], inv_freq=10000.0 ** (-torch.arange(0, c["rot"], 2, device=DEV, dtype=torch.float64) / c["rot"]),
             positions=torch.from_numpy(rng.integers(0, 32768, n).astype(np.int32)).to(DEV), eps=1e-6, wq=None, wk=None)
    if c["norm"]:
        s["wq"], s["wk"] = (1.0 + 0.2 * torch.randn(D, device=DEV, generator=g) for _ in range(2))
    names = ["out_q", "out_k"]
    if c["train"]:
        s["dy_q"], s["dy_k"] = (torch.randn(n, h, D, device=DEV, generator=g).to(dt) for h in (Hq, Hk))
        names += ["dx_q", "dx_k"]
        s["dw_q"], s["dw_k"] = (torch.empty(D, device=DEV) if c["norm"] else None for _ in range(2))
    for name in names:
        s[name] = torch.empty(n, Hq if name.endswith("q") else Hk, D, device=DEV, dtype=dt)
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms


def _plain_attention(s):
    T, Hq, Hkv, D = (s[k] for k in ("T", "Hq", "Hkv", "D"))
    # one row more than there are tokens: what the padded places read and write
    pad = lambda x: torch.cat([x.float(), torch.zeros_like(x[:1], dtype=torch.float32)])  # noqa: E731
    q, k, v = pad(s["q"]), pad(s["k"]), pad(s["v"])
    dout = pad(s["dout"]) if s["train"] else None
    got = {"out": torch.empty(T + 1, Hq, D, device=DEV), "lse": torch.empty(T + 1, Hq, device=DEV)}
    if s["train"]:
        got.update(dq=torch.empty(T + 1, Hq, D, device=DEV), dk=torch.zeros(T + 1, Hkv, D, device=DEV), dv=torch.zeros(T + 1, Hkv, D, device=DEV))
    off, N = s["offsets"], s["N"]
    place = torch.arange(N, device=DEV) if s["group_offsets"] is None else s["group_offsets"][:-1] + torch.arange(N, device=DEV)
    own_p = _tokens(off[place], off[place + 1], s["prompt_max"], T)
    _plain_pass(s, q, k, v, dout, got, own_p, own_p[:, :0])
    if s["R"]:
        r = torch.arange(s["R"], device=DEV)
        group = torch.searchsorted(s["group_offsets"], r, right=True) - 1
        place = r + group + 1
        _plain_pass(s, q, k, v, dout, got, _tokens(off[place], off[place + 1], s["rollout_max"], T), own_p[group])
    return {name: x[:T].to(torch.float32 if name == "lse" else s["q"].dtype) for name, x in got.items()}


def _tokens(lo, hi, width, T):
    """Places of the sequences' tokens, [sequences, width]; T where a sequence is shorter."""
    at = lo[:, None] + torch.arange(width, device=DEV)
    return torch.where(at < hi[:, None], at, torch.full_like(at, T))


def _plain_pass(s, q, k, v, dout, got, mine, shared):
    """Sequences of the tokens `mine` [n, L] over the keys of the tokens `shared` [n, P] and their own."""
    T, Hq, Hkv, D, g = s["T"], s["Hq"], s["Hkv"], s["D"], s["Hq"] // s["Hkv"]
    n, L = mine.shape
    keys = torch.cat([shared, mine], 1)
    K = keys.shape[1]
    hidden = (keys == T)[:, None, :].expand(n, L, K).clone()
    if s["causal"]:
        hidden[:, :, K - L:] |= torch.ones(L, L, device=DEV, dtype=torch.bool).triu(1)
    rows = lambda x: x[mine].reshape(n, L, Hkv, g, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, g * L, D)  # noqa: E731
    back = lambda x: x.reshape(n, Hkv, g, L, x.shape[-1]).permute(0, 3, 1, 2, 4).reshape(n * L, Hq, x.shape[-1])  # noqa: E731
    qs, ks, vs = rows(q), k[keys].permute(0, 2, 1, 3), v[keys].permute(0, 2, 1, 3)
    p = torch.matmul(qs, ks.transpose(-1, -2)).mul_(s["scale"]).reshape(n, Hkv, g, L, K)
    p.masked_fill_(hidden[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, torch.ones_like(total))).reshape(n, Hkv, g * L, K)
    o = torch.matmul(p, vs)
    to = mine.reshape(-1)
    got["out"][to] = back(o)
    got["lse"][to] = back((m + torch.log(total)).reshape(n, Hkv, g * L, 1))[..., 0]
    if not s["train"]:
        return
    do = rows(dout)
    from_ = keys.reshape(-1)
    got["dv"].index_add_(0, from_, torch.matmul(p.transpose(-1, -2), do).permute(0, 2, 1, 3).reshape(n * K, Hkv, D))
    ds = torch.matmul(do, vs.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    del p
    got["dq"][to] = back(torch.matmul(ds, ks)) * s["scale"]
    got["dk"].index_add_(0, from_, torch.matmul(ds.transpose(-1, -2), qs).permute(0, 2, 1, 3).reshape(n * K, Hkv, D) * s["scale"])


def _turn(x, cos, sin, pairs, rot):
    """The first `rot` values of each row turned by the angles, two at a time."""
    y = x[..., :rot]
    if pairs:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_rotate(s):
    angle = (s["positions"].double()[:, None] * s["inv_freq"])[:, None, :]        # in 64 bits: far positions make large angles
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q = _plain_rotate_one(s, s["q"], s["wq"], cos, sin, s.get("dy_q"))
    k = _plain_rotate_one(s, s["k"], s["wk"], cos, sin, s.get("dy_k"))
    return {name + tail: x for tail, y in (("_q", q), ("_k", k)) for name, x in y.items()}


def _plain_rotate_one(s, x, w, cos, sin, dy):
    dt, x = x.dtype, x.float()
    z = x
    if w is not None:
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"])
        z = x * r * w
    got = {"out": _turn(z, cos, sin, s["pairs"], s["rot"]).to(dt)}
    if s["train"]:
        g = _turn(dy.float(), cos, -sin, s["pairs"], s["rot"])
        dx = g
        if w is not None:
            got["dw"] = (x * r * g).sum((0, 1), dtype=torch.float64).float()
            wg = w * g
            dx = r * (wg - x * r * (x * r * wg).mean(-1, keepdim=True))
        got["dx"] = dx.to(dt)
    return got


# ---------------------------------------------------------------------------------------------------------------
# through the library


def _own_attention(s):
    from paper_2605_07114_b200 import hora
    if "op_handle" not in s:
        s["op_handle"] = hora.PackedAttention(s["offsets"], s["T"], s["Hq"], s["Hkv"], s["D"], TYPES[s["dtype"]], group_offsets=s["group_offsets"],
                                              causal=s["causal"], sm_scale=s["scale"], backward=s["train"])
    out, lse = s["op_handle"].run(s["q"], s["k"], s["v"])
    if not s["train"]:
        return {"out": out, "lse": lse}
    dq, dk, dv = s["op_handle"].backward(s["q"], s["k"], s["v"], out, lse, s["dout"])
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _own_rotate(s):
    from paper_2605_07114_b200 import hora
    if "op_handle" not in s:
        s["op_handle"] = hora.QkRotation(s["inv_freq"], s["D"], q_weight=s["wq"], k_weight=s["wk"], eps=s["eps"],
                                         layout=hora.ROTATE_PAIRS if s["pairs"] else hora.ROTATE_HALVES)
    s["op_handle"].run(s["q"], s["k"], s["positions"], s["out_q"], s["out_k"])
    got = {"out_q": s["out_q"], "out_k": s["out_k"]}
    if s["train"]:
        s["op_handle"].backward(s["dy_q"], s["dy_k"], s["q"], s["k"], s["positions"], s["dx_q"], s["dx_k"], s["dw_q"], s["dw_k"])
        got.update(dx_q=s["dx_q"], dx_k=s["dx_k"])
        if s["norm"]:
            got.update(dw_q=s["dw_q"], dw_k=s["dw_k"])
    return got


def run(state):
    if state["op"] == "attention":
        return _own_attention(state) if own else _plain_attention(state)
    return _own_rotate(state) if own else _plain_rotate(state)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    c = case
    size = BYTES[c["dtype"]]
    if c["op"] == "rotate":
        values = c["n"] * (c["Hq"] + c["Hk"]) * c["D"]
        # forward: x in, y out; backward: the gradient and (for the norm) x again in, its gradient out
        return {"bytes": float(values * size * (2 + (2 + bool(c["norm"]) if c["train"] else 0)) + 4 * c["n"]), "flops": 0.0}
    # a prompt is on average three quarters, a rollout half as long as the longest; squares of such lengths are 7/12 and 1/3 of its square;
    # one of an odd number is the longest
    P, L, N, R = c["prompt"], c["rollout"], c["N"], c["R"]
    prompts, prompts2 = (N - N % 2) * 0.75 * P + N % 2 * P, ((N - N % 2) * 7 / 12 + N % 2) * P * P
    rollouts, rollouts2 = (R - R % 2) * 0.5 * L + R % 2 * L, ((R - R % 2) / 3 + R % 2) * L * L
    tokens = prompts + rollouts
    half = 0.5 if c["causal"] else 1.0
    pairs = half * prompts2 + rollouts * prompts / N + half * rollouts2
    rows = tokens * c["D"] * size
    moved = rows * (2 * c["Hq"] + 2 * c["Hkv"]) + tokens * c["Hq"] * 4
    if c["train"]:       # the gradient of the output and what the forward pass left in, the gradients of queries, keys and values out
        moved += rows * (4 * c["Hq"] + 4 * c["Hkv"]) + tokens * c["Hq"] * 4
    return {"bytes": float(moved), "flops": 2.0 * c["D"] * c["Hq"] * pairs * (7 if c["train"] else 2)}


# ---------------------------------------------------------------------------------------------------------------
# the definitions, in 64 bits, one sequence or one part of the rows at a time


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_attention(s) if s["op"] == "attention" else _exact_rotate(s)


def _exact_attention(s):
    T, Hq, Hkv, D = (s[k] for k in ("T", "Hq", "Hkv", "D"))
    g = Hq // Hkv
    off = s["offsets"].tolist()
    go = s["group_offsets"].tolist() if s["R"] else list(range(s["N"] + 1))
    prompt_of = {}
    if s["R"]:
        for i in range(s["N"]):
            for r in range(go[i], go[i + 1]):
                prompt_of[r + i + 1] = go[i] + i
    new = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device=DEV)  # noqa: E731
    out, lse, dq, dk, dv = new(T, Hq, D), new(T, Hq), new(T, Hq, D), new(T, Hkv, D), new(T, Hkv, D)
    for i in range(len(off) - 1):
        a, b = off[i], off[i + 1]
        at = torch.arange(a, b, device=DEV)
        if i in prompt_of:
            j = prompt_of[i]
            at = torch.cat([torch.arange(off[j], off[j + 1], device=DEV), at])
        k, v = s["k"][at].double().transpose(0, 1), s["v"][at].double().transpose(0, 1)             # [Hkv, keys, D]
        step = max(1, (1 << 28) // (Hq * at.numel()))
        for c in range(a, b, step):
            e = min(b, c + step)
            q = s["q"][c:e].double().reshape(e - c, Hkv, g, D).permute(1, 2, 0, 3)                   # [Hkv, g, rows, D]
            z = torch.einsum("hgtd,hkd->hgtk", q, k) * s["scale"]
            if s["causal"]:
                z.masked_fill_(at[None, :] > torch.arange(c, e, device=DEV)[:, None], -math.inf)
            top = torch.logsumexp(z, -1, keepdim=True)
            p = torch.exp(z - top)
            o = torch.einsum("hgtk,hkd->hgtd", p, v)
            out[c:e] = o.permute(2, 0, 1, 3).reshape(e - c, Hq, D)
            lse[c:e] = top[..., 0].permute(2, 0, 1).reshape(e - c, Hq)
            if s["train"]:
                do = s["dout"][c:e].double().reshape(e - c, Hkv, g, D).permute(1, 2, 0, 3)
                dv.index_add_(0, at, torch.einsum("hgtk,hgtd->khd", p, do))
                dz = p * (torch.einsum("hgtd,hkd->hgtk", do, v) - (do * o).sum(-1, keepdim=True)) * s["scale"]
                dq[c:e] = torch.einsum("hgtk,hkd->hgtd", dz, k).permute(2, 0, 1, 3).reshape(e - c, Hq, D)
                dk.index_add_(0, at, torch.einsum("hgtk,hgtd->khd", dz, q))
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv} if s["train"] else {"out": out, "lse": lse}


def _exact_rotate(s):
    got = {}
    rot = s["rot"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), (s["positions"].double()[:, None] * s["inv_freq"])[:, None, :])

    def rotate(x, by):       # as complex numbers
        y = x[..., :rot]
        y = y.unflatten(-1, (-1, 2)) if s["pairs"] else y.unflatten(-1, (2, -1)).transpose(-1, -2)
        y = torch.view_as_real(torch.view_as_complex(y.contiguous()) * by)
        return torch.cat([(y if s["pairs"] else y.transpose(-1, -2)).flatten(-2), x[..., rot:]], -1)

    for tail, w in (("_q", s["wq"]), ("_k", s["wk"])):
        x = s[tail[1:]].double()
        norm = torch.sqrt((x ** 2).mean(-1, keepdim=True) + s["eps"]) if w is not None else 1.0
        u = x / norm
        got["out" + tail] = rotate(u * w.double() if w is not None else u, turn)
        if s["train"]:
            d = rotate(s["dy" + tail].double(), turn.conj())
            if w is not None:
                got["dw" + tail] = (u * d).sum((0, 1))
                d = d * w.double()
                d = (d - u * (u * d).mean(-1, keepdim=True)) / norm
            got["dx" + tail] = d
    return got
