"""The operators of a rollout decode step, as cases to be measured.

One decode step of a batch of rollout groups: the new keys and values go into a paged (and quantised) cache, the
queries of every rollout attend to their prompt's cache, shared by the group, and to the rollout's own, and drafted
tokens are verified against the target's probabilities.  ``run`` makes one pass through one of these operators:
in plain torch operations where ``own`` is false, through the library where it is true.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
F8 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": F8}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
GRID = 2.0 ** 38          # probabilities are held on the grid 2^-38 when a token is drawn from them


def _attention(name, N, R, T, Hq, Hkv, D, prefix, suffix, dtype, cache, page):
    c = dict(op="attention", N=N, R=R, T=T, Hq=Hq, Hkv=Hkv, D=D, prefix=prefix, suffix=suffix, dtype=dtype, cache=cache, page=page)
    return dict(c, name=name) if name else c


def _cache(name, n, H, D, dtype, cache, page, out):
    c = dict(op="cache", n=n, H=H, D=D, dtype=dtype, cache=cache, page=page, out=out)
    return dict(c, name=name) if name else c


def _verify(name, R, K, V, dtype, rows):
    c = dict(op="verify", R=R, K=K, V=V, dtype=dtype, rows=rows)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the first tokens of one prompt's pre-rollouts: eight rollouts, hardly any cache of their own; latency counts
        _attention("attn one prompt G0=8", 1, 8, 1, 12, 2, 128, 211, 24, "bf16", "bf16", 16),
        # one shard of a training step: 15 prompts, 480 rollouts in groups of uneven size, responses up to 2048 tokens
        _attention("attn shard 15x32", 15, 480, 1, 28, 4, 128, 413, 2048, "bf16", "bf16", 16),
        # a whole training batch on one GPU: 60 prompts, 1920 rollouts, the quantised cache
        _attention("attn batch 60x32 e4m3", 60, 1920, 1, 16, 2, 128, 509, 1536, "bf16", "e4m3", 32),
        # a few long problems (documents, tool traces) with wide groups: the shared part outweighs the rollouts' own
        _attention("attn long prefix fp16", 4, 96, 1, 32, 8, 128, 32749, 701, "f16", "f16", 64),
        # one verification pass: up to four drafted tokens and the last sampled one of each rollout, smaller heads
        _attention("attn drafts T=5 D=64", 16, 256, 5, 16, 4, 64, 1531, 1021, "bf16", "bf16", 16),
        # very wide groups over a long prompt, hundreds of query rows to a key: bound by products, not by bytes
        _attention("attn wide groups", 2, 512, 2, 64, 8, 128, 8192, 257, "bf16", "bf16", 128),
        # one decode step's new keys and values
        _cache("cache step e4m3", 480, 4, 128, "bf16", "e4m3", 16, "bf16"),
        # the prompts of a batch, all layers' worth of tokens in one go
        _cache("cache prompts e4m3", 131072, 8, 128, "bf16", "e4m3", 64, "bf16"),
        # keys and values from a 32-bit layer, a ragged number of tokens, smaller heads
        _cache("cache f32 ragged", 50021, 5, 64, "f32", "e4m3", 16, "f16"),
        # one prompt's rollouts with four drafts each
        _verify("verify 8x4", 8, 4, 32000, "f32", True),
        # one shard's rollouts over a large vocabulary
        _verify("verify 480x4", 480, 4, 151936, "f32", True),
        # drafts looked up in the other rollouts of the group (no probabilities of their own), odd vocabulary, 16-bit rows
        _verify("verify lookup bf16", 1920, 3, 50257, "bf16", False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed() if c["op"] == "attention")
    while True:
        op = rng.choice(["attention", "attention", "cache", "verify"])
        if op == "attention":
            N = _log(rng, 1, 64)
            Hkv = rng.choice([1, 2, 3, 4, 8])
            T = rng.choice([1, 1, 1, 2, 3, 5, 8])
            dtype = rng.choice(["bf16", "f16"])
            c = _attention(None, N, N * _log(rng, 1, 64) + rng.randrange(N), T, Hkv * rng.choice([1, 3, 4, 5, 7, 8]), Hkv, rng.choice([64, 128, 128]),
                           _log(rng, 16, 32768), max(T, _log(rng, 4, 4096)), dtype, rng.choice([dtype, dtype, "e4m3"]), rng.choice([16, 32, 64, 128]))
        elif op == "cache":
            dtype = rng.choice(["bf16", "f16", "f32"])
            out = rng.choice(["bf16", "f16", "f32"])
            c = _cache(None, _log(rng, 1, 131072), rng.randint(1, 8), rng.choice([64, 128]), dtype,
                       rng.choice(["e4m3", "e4m3", "bf16" if dtype == "f32" else dtype]), rng.choice([16, 32, 64, 128]), out)
        else:
            c = _verify(None, _log(rng, 1, 1024), rng.randint(0, 8), _log(rng, 1000, 200000), rng.choice(["f32", "f32", "bf16", "f16"]), rng.random() < 0.6)
            if c["R"] * (2 * c["K"] + 1) * c["V"] > 480 * 9 * 151936:
                continue
        if _cost(c) <= (most if op == "attention" else max(_cost(x) for x in listed() if x["op"] == op)):
            return c


def _cost(c):
    """Roughly the time of a pass in its plain form, to keep drawn cases within the listed ones."""
    if c["op"] == "attention":
        keys = c["N"] * c["prefix"] + c["R"] * c["suffix"]
        products = c["R"] * c["T"] * c["Hq"] * (c["prefix"] + c["suffix"])
        return keys * c["Hkv"] * c["D"] * 40 + products * (c["D"] + 40)
    if c["op"] == "cache":
        return c["n"] * c["H"] * c["D"]
    return c["R"] * c["V"]


# ---------------------------------------------------------------------------------------------------------------
# inputs


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g, np.random.Generator(np.random.PCG64(seed))


def _pages(rng, lengths, page):
    """A table of page numbers for sequences of these lengths, pages in no order, as an allocator leaves them after a while."""
    need = -(-lengths // page)
    total = int(need.sum()) + 3
    order = rng.permutation(total).astype(np.int32)
    table = np.zeros((len(lengths), max(1, int(need.max()))), np.int32)
    ends = np.cumsum(need)
    for i, (e, n) in enumerate(zip(ends, need)):
        table[i, :n] = order[e - n:e]
    return table, total


def _row_exponent(x):
    """Per row of x: the least e with max|x| / 2^e <= 448 over the finite values (0 for a row of zeros)."""
    a = x.float().abs()
    a = torch.where(torch.isfinite(a), a, torch.zeros_like(a)).amax(-1)
    m, e = torch.frexp(a)                                     # a = m 2^e, 1/2 <= m < 1;  448 = 0.875 * 2^9
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(a > 0, e, torch.zeros_like(e)).clamp(-126, 127)


def _quantise(x):
    """(codes, exponent bytes): e4m3 values of x / 2^e, and e + 127."""
    e = _row_exponent(x)
    y = torch.ldexp(x.float(), -e.unsqueeze(-1)).clamp(-448.0, 448.0)
    return y.to(F8), (e + 127).to(torch.uint8)


def _value(codes, exps):
    return torch.ldexp(codes.float(), (exps.to(torch.int32) - 127).unsqueeze(-1))


def prepare(case, seed):
    g, rng = _generator(seed)
    return {"attention": _prepare_attention, "cache": _prepare_cache, "verify": _prepare_verify}[case["op"]](dict(case), g, rng)


def _prepare_attention(c, g, rng):
    N, R, T, Hq, Hkv, D, page = (c[k] for k in ("N", "R", "T", "Hq", "Hkv", "D", "page"))
    sizes = 1 + rng.multinomial(R - N, rng.dirichlet(np.full(N, 2.0)))          # uneven groups, as the allocation makes them
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    q_len = rng.integers(1, T + 1, R).astype(np.int32)
    prefix_len = rng.integers(max(1, c["prefix"] // 2), c["prefix"] + 1, N).astype(np.int32)
    suffix_len = np.maximum(rng.integers(1, c["suffix"] + 1, R), q_len).astype(np.int32)
    table, n_pages = _pages(rng, np.concatenate([prefix_len, suffix_len]), page)
    n_prefix, n_suffix = -(-int(prefix_len.max()) // page), -(-int(suffix_len.max()) // page)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    dt = TYPES[c["dtype"]]
    # queries larger than keys: some positions matter, most do not
    q = (2.0 * torch.randn(R, T, Hq, D, device=DEV, generator=g)).to(dt)
    s = dict(c, q=q, off=t(off), q_len=t(q_len), prefix_len=t(prefix_len), suffix_len=t(suffix_len),
             prefix_pages=t(table[:N, :n_prefix]), suffix_pages=t(table[N:, :n_suffix]), n_pages=n_pages, g_max=int(sizes.max()), scale=D ** -0.5)
    for name in ("k", "v"):
        x = torch.randn(n_pages, Hkv, page, D, device=DEV, generator=g, dtype=torch.float32 if c["cache"] == "e4m3" else dt)
        s[name], s[name + "_exp"] = _quantise(x) if c["cache"] == "e4m3" else (x, None)
    return s


def _prepare_cache(c, g, rng):
    n, H, D, page = (c[k] for k in ("n", "H", "D", "page"))
    # keys and values side by side, as one projection writes them; a few channels are much larger than the others
    kv = torch.randn(n, 2, H, D, device=DEV, generator=g)
    kv = (kv * torch.exp(torch.randn(2, H, D, device=DEV, generator=g))).to(TYPES[c["dtype"]])
    n_pages = -(-n // page) + 2
    order = rng.permutation(n_pages).astype(np.int64)
    at = np.arange(n, dtype=np.int64)
    slots = torch.from_numpy(order[at // page] * page + at % page).to(DEV)
    s = dict(c, k_in=kv[:, 0], v_in=kv[:, 1], slots=slots, n_pages=n_pages)
    for name in ("k", "v"):
        s[name] = torch.zeros(n_pages, H, page, D, device=DEV, dtype=torch.float32).to(TYPES[c["cache"]])
        s[name + "_exp"] = torch.full((n_pages, H, page), 127, device=DEV, dtype=torch.uint8) if c["cache"] == "e4m3" else None
        s[name + "_out"] = torch.empty(n, H, D, device=DEV, dtype=TYPES[c["out"]])
    return s


def _prepare_verify(c, g, rng):
    R, K, V = c["R"], c["K"], c["V"]
    dt = TYPES[c["dtype"]]
    # a draft model's scores are the target's with some noise: most drafts are accepted
    logits = 2.5 * torch.randn(R, K + 1, V, device=DEV, generator=g)
    target = torch.softmax(logits, -1).to(dt)
    draft = None
    if K and c["rows"]:
        draft = torch.softmax(logits[:, :K] + 0.5 * torch.randn(R, K, V, device=DEV, generator=g), -1).to(dt)
    tokens = torch.empty(R, K, device=DEV, dtype=torch.int32)
    for k in range(K):      # drafts drawn from the draft's probabilities, or from the target's where there are none
        p = (target if draft is None else draft)[:, k].float()
        tokens[:, k] = (p / torch.empty_like(p).exponential_(generator=g).clamp_min(1e-20)).argmax(-1).to(torch.int32)
    del logits
    return dict(c, target=target, draft=draft, tokens=tokens,
                length=torch.from_numpy(rng.integers(max(0, K - 1), K + 1, R).astype(np.int32)).to(DEV),
                u_accept=torch.rand(R, K, device=DEV, generator=g), u_sample=torch.rand(R, device=DEV, generator=g),
                n_accepted=torch.empty(R, device=DEV, dtype=torch.int32), out=torch.empty(R, K + 1, device=DEV, dtype=torch.int32))


# ---------------------------------------------------------------------------------------------------------------
# plain forms


def _keys(s, name, table):
    """The cached rows of a page table, [sequences, Hkv, table width * page, D] in 32 bits."""
    x = s[name][table.long()]
    x = x.float() if s[name + "_exp"] is None else _value(x, s[name + "_exp"][table.long()])
    n, w, H, page, D = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, H, w * page, D)


def _plain_attention(s):
    N, R, T, Hq, Hkv, D = (s[k] for k in ("N", "R", "T", "Hq", "Hkv", "D"))
    g, G = Hq // Hkv, s["g_max"]
    r = torch.arange(R, device=DEV)
    group = torch.searchsorted(s["off"], r, right=True) - 1
    place = r - s["off"][group]
    member = (s["off"][:-1, None] + torch.arange(G, device=DEV)).clamp_max(R - 1)
    q = s["q"].float().reshape(R, T, Hkv, g, D).permute(0, 2, 1, 3, 4)                      # [R, Hkv, T, g, D]
    rows = T * g

    def to_groups(x):       # [R, Hkv, rows, X] -> [N, Hkv, G * rows, X]
        return x[member].permute(0, 2, 1, 3, 4).reshape(N, Hkv, G * rows, x.shape[-1])

    def to_rollouts(x):     # and back
        return x.reshape(N, Hkv, G, rows, x.shape[-1]).permute(0, 2, 1, 3, 4)[group, place]

    q = q.reshape(R, Hkv, rows, D)
    shared = to_rollouts(torch.matmul(to_groups(q), _keys(s, "k", s["prefix_pages"]).transpose(-1, -2))) * s["scale"]
    at = torch.arange(shared.shape[-1], device=DEV)
    shared.masked_fill_((at >= s["prefix_len"][group][:, None])[:, None, None, :], -math.inf)
    single = torch.matmul(q, _keys(s, "k", s["suffix_pages"]).transpose(-1, -2)) * s["scale"]
    at = torch.arange(single.shape[-1], device=DEV)
    last = (s["suffix_len"] - s["q_len"])[:, None] + torch.arange(T, device=DEV)            # the query's own position
    hidden = (at > last[:, :, None]) | (torch.arange(T, device=DEV) >= s["q_len"][:, None])[:, :, None]
    single = single.reshape(R, Hkv, T, g, -1).masked_fill_(hidden[:, None, :, None, :], -math.inf).reshape(R, Hkv, rows, -1)
    pad = (torch.arange(T, device=DEV) >= s["q_len"][:, None])[:, None, :, None].expand(R, Hkv, T, g).reshape(R, Hkv, rows, 1)
    shared.masked_fill_(pad, -math.inf)
    m = torch.maximum(shared.amax(-1, keepdim=True), single.amax(-1, keepdim=True))
    m0 = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    shared, single = torch.exp(shared - m0), torch.exp(single - m0)
    total = shared.sum(-1, keepdim=True) + single.sum(-1, keepdim=True)
    o = to_rollouts(torch.matmul(to_groups(shared), _keys(s, "v", s["prefix_pages"]))) + torch.matmul(single, _keys(s, "v", s["suffix_pages"]))
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = m + torch.log(total)
    o = o.reshape(R, Hkv, T, g, D).permute(0, 2, 1, 3, 4).reshape(R, T, Hq, D)
    return {"out": o.to(s["q"].dtype), "lse": lse.reshape(R, Hkv, T, g).permute(0, 2, 1, 3).reshape(R, T, Hq)}


def _plain_cache(s):
    page, slots = s["page"], s["slots"]
    p, i = slots // page, slots % page
    got = {}
    for name in ("k", "v"):
        x = s[name + "_in"]
        if s["cache"] == "e4m3":
            codes, exps = _quantise(x)
            s[name].view(torch.uint8)[p, :, i] = codes.view(torch.uint8)
            s[name + "_exp"][p, :, i] = exps
            y = _value(s[name].view(torch.uint8)[p, :, i].view(F8), s[name + "_exp"][p, :, i])
        else:
            s[name][p, :, i] = x.to(s[name].dtype)
            y = s[name][p, :, i]
        got[name] = y.to(TYPES[s["out"]])
    return got


def _plain_verify(s):
    R, K, V = s["R"], s["K"], s["V"]
    r = torch.arange(R, device=DEV)
    if K:
        x = s["tokens"].long().unsqueeze(-1)
        # the product of two 24-bit numbers is exact in 64 bits: the comparison depends on no rounding
        p = s["target"][:, :K].gather(-1, x).squeeze(-1).double()
        q = torch.ones_like(p) if s["draft"] is None else s["draft"].gather(-1, x).squeeze(-1).double()
        ok = (s["u_accept"].double() * q < p) & (torch.arange(K, device=DEV) < s["length"][:, None])
        n = ok.long().cumprod(-1).sum(-1)
        refused = n < s["length"]
        j = n.clamp_max(K - 1)
    else:
        n, refused = torch.zeros(R, device=DEV, dtype=torch.long), torch.zeros(R, device=DEV, dtype=torch.bool)
    grid = (s["target"][r, n].float() * GRID).long()
    weight = grid
    if K:
        if s["draft"] is None:
            minus = torch.zeros_like(grid).scatter_(1, s["tokens"][r, j].long().unsqueeze(-1), int(GRID))
        else:
            minus = (s["draft"][r, j].float() * GRID).long()
        rest = torch.where(refused[:, None], grid - minus, grid).clamp_min(0)
        weight = torch.where(rest.sum(-1, keepdim=True) > 0, rest, grid)
    total = weight.sum(-1)
    u = (s["u_sample"] * 2.0 ** 24).long().clamp(0, (1 << 24) - 1)
    limit = (total >> 24) * u + (((total & 0xFFFFFF) * u) >> 24)
    token = (weight.cumsum(-1) <= limit[:, None]).sum(-1)
    at = torch.arange(K + 1, device=DEV)
    drafts = torch.cat([s["tokens"].long(), torch.full((R, 1), -1, device=DEV)], 1)
    out = torch.where(at < n[:, None], drafts, torch.where(at == n[:, None], token[:, None], torch.full_like(drafts, -1)))
    return {"n_accepted": n.to(torch.int32), "tokens": out.to(torch.int32)}


# ---------------------------------------------------------------------------------------------------------------
# through the library


def _own_attention(s):
    from paper_2605_07114_b200 import hora
    if "op_handle" not in s:
        cache = hora.PagedCache.over(s["k"], s["v"], s["k_exp"], s["v_exp"])
        s["op_handle"] = hora.GroupAttention(cache, s["Hq"], s["T"], TYPES[s["dtype"]], group_offsets=s["off"],
                                             prefix_pages=s["prefix_pages"], prefix_len=s["prefix_len"],
                                             suffix_pages=s["suffix_pages"], suffix_len=s["suffix_len"], q_len=s["q_len"], sm_scale=s["scale"])
    out, lse = s["op_handle"].run(s["q"])
    return {"out": out, "lse": lse}


def _own_cache(s):
    from paper_2605_07114_b200 import hora
    if "op_handle" not in s:
        s["op_handle"] = hora.PagedCache.over(s["k"], s["v"], s["k_exp"], s["v_exp"])
    s["op_handle"].write(s["k_in"], s["v_in"], s["slots"])
    s["op_handle"].read(s["slots"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_verify(s):
    from paper_2605_07114_b200 import hora
    hora.hora_verify_drafts(s["target"], s["draft"], s["tokens"], s["length"], s["R"], s["K"], s["V"], s["u_accept"], s["u_sample"], s["n_accepted"], s["out"])
    return {"n_accepted": s["n_accepted"], "tokens": s["out"]}


def run(state):
    op = state["op"]
    if op == "attention":
        return _own_attention(state) if own else _plain_attention(state)
    if op == "cache":
        return _own_cache(state) if own else _plain_cache(state)
    return _own_verify(state) if own else _plain_verify(state)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    c = case
    if c["op"] == "attention":
        # on average three quarters of the prefix and half of the suffix are filled; half of the query slots (T > 1) hold one
        queries = c["R"] * (c["T"] + 1) / 2
        prefix, suffix = 0.75 * c["prefix"], 0.5 * c["suffix"]
        row = 2 * c["Hkv"] * (c["D"] * BYTES[c["cache"]] + (c["cache"] == "e4m3"))
        moved = (c["N"] * prefix + c["R"] * suffix) * row + queries * c["Hq"] * c["D"] * 2 + c["R"] * c["T"] * c["Hq"] * (c["D"] * 2 + 4)
        return {"bytes": moved, "flops": 4.0 * c["D"] * c["Hq"] * queries * (prefix + suffix)}
    if c["op"] == "cache":
        kept = c["D"] * BYTES[c["cache"]] + (c["cache"] == "e4m3")
        return {"bytes": 2.0 * c["n"] * c["H"] * (c["D"] * (BYTES[c["dtype"]] + BYTES[c["out"]]) + 2 * kept) + 16.0 * c["n"], "flops": 0.0}
    # the row the new token is drawn from, and the draft's row beside it (for the rollouts that refuse a draft)
    return {"bytes": float(c["R"]) * c["V"] * BYTES[c["dtype"]] * (2 if c["rows"] and c["K"] else 1) + 16.0 * c["R"] * (c["K"] + 1), "flops": 0.0}


# ---------------------------------------------------------------------------------------------------------------
# the definitions, in 64 bits, one sequence at a time


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "cache": _exact_cache, "verify": _exact_verify}[case["op"]](s)


def _exact_attention(s):
    R, T, Hq, Hkv, D, page = (s[k] for k in ("R", "T", "Hq", "Hkv", "D", "page"))
    off, pl, sl, ql = (s[k].tolist() for k in ("off", "prefix_len", "suffix_len", "q_len"))
    out = torch.zeros(R, T, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.full((R, T, Hq), -math.inf, dtype=torch.float64, device=DEV)

    def rows(name, pages, n):
        ids = pages[:-(-n // page)].long()
        x = s[name][ids].float().double()
        if s[name + "_exp"] is not None:
            x = x * torch.exp2(s[name + "_exp"][ids].double() - 127.0)[..., None]
        return x.transpose(1, 2).reshape(-1, Hkv, D)[:n].transpose(0, 1)          # [Hkv, n, D]

    for i in range(s["N"]):
        kp, vp = (rows(name, s["prefix_pages"][i], pl[i]) for name in ("k", "v"))
        for r in range(off[i], off[i + 1]):
            ks, vs = (rows(name, s["suffix_pages"][r], sl[r]) for name in ("k", "v"))
            q = s["q"][r, :ql[r]].double().reshape(ql[r], Hkv, Hq // Hkv, D).transpose(0, 1)   # [Hkv, t, g, D]
            for t in range(ql[r]):
                seen = sl[r] - ql[r] + t + 1
                z = s["scale"] * torch.cat([q[:, t] @ kp.transpose(1, 2), q[:, t] @ ks[:, :seen].transpose(1, 2)], -1)
                e = torch.logsumexp(z, -1, keepdim=True)
                p = torch.exp(z - e)
                out[r, t] = (p[..., :pl[i]] @ vp + p[..., pl[i]:] @ vs[:, :seen]).reshape(Hq, D)
                lse[r, t] = e.reshape(Hq)
    return {"out": out, "lse": lse}


def _exact_cache(s):
    got = {}
    for name in ("k", "v"):
        x = s[name + "_in"].double()
        if s["cache"] == "e4m3":
            top = x.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 448.0))
            e = torch.where(top / torch.exp2(e) > 448.0, e + 1, torch.where(top / torch.exp2(e - 1) <= 448.0, e - 1, e))
            scale = torch.exp2(e)
            y = x / scale
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3.0)   # spacing of 4-bit significands, fixed below 2^-6
            x = torch.round(y / step) * step * scale
        else:
            x = x.to(TYPES[s["cache"]]).double()
        got[name] = x.to(TYPES[s["out"]]).double()
    return got


def _exact_verify(s):
    R, K, V = s["R"], s["K"], s["V"]
    tokens, length = s["tokens"].cpu().numpy(), s["length"].tolist()
    ua, us = s["u_accept"].double().cpu().numpy(), s["u_sample"].double().tolist()
    n_accepted, out = np.zeros(R, np.int32), np.full((R, K + 1), -1, np.int32)
    for r in range(R):
        n = 0
        while n < length[r]:
            x = int(tokens[r, n])
            q = 1.0 if s["draft"] is None else float(s["draft"][r, n, x])
            if not ua[r, n] * q < float(s["target"][r, n, x]):
                break
            n += 1
        p = np.floor(s["target"][r, n].double().cpu().numpy() * GRID)
        w = p
        if n < length[r]:
            q = np.floor(s["draft"][r, n].double().cpu().numpy() * GRID) if s["draft"] is not None else np.where(np.arange(V) == tokens[r, n], GRID, 0.0)
            w = np.maximum(p - q, 0.0)
            w = w if w.any() else p
        sums = np.cumsum(w.astype(np.int64))
        limit = int(sums[-1]) * int(us[r] * 2 ** 24) >> 24
        n_accepted[r] = n
        out[r, :n] = tokens[r, :n]
        out[r, n] = int(np.searchsorted(sums, limit, side="right"))
    return {"n_accepted": n_accepted, "tokens": out}
