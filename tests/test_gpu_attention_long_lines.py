"""hora_group_attention where one sequence has more steps (blocks of rows by keys by heads) than 32 bits count.

The long prompt is one page of keys named over and over, so that its softmax is that of the page.  What counts is the sequences behind
it: their place on the line of steps follows from the long one's number of steps.

Tolerance.  The short group's: weights in fp16 (2^-11 relative, 2^-25 of the largest value below the normal range), bf16 output (2^-8), scores
as fp32 sums (below 2^-10 here).  The long group's: sums of 2^17 weights in fp32 one after the other and of 2^16 products, each off by at most 2^-24 and
2^-23 relative to the sum: 2^-7 each."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda"


@pytest.mark.parametrize("pages_of_prompt", [128, 8192])
def test_sequences_behind_a_very_long_line_are_where_the_plan_says(pages_of_prompt):
    from paper_2605_07114_b200 import hora
    R1, R2, Hq, Hkv, D, page, P2, own = 2100, 3, 256, 32, 64, 128, 50, 5
    steps = pages_of_prompt * (page // 32) * R1 * Hkv                     # eight rows of a rollout and cache head to a block, 32 keys to a step
    assert pages_of_prompt < 8192 or steps > 2 ** 31
    c = hora.PagedCache.empty(3, page, Hkv, D, torch.float8_e4m3fn)
    g = torch.Generator(device=DEV).manual_seed(9)
    n = 3 * page
    slots = torch.arange(n, device=DEV)
    c.write(*(torch.randn(n, Hkv, D, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2)), slots)
    k, v = (torch.empty(n, Hkv, D, device=DEV) for _ in range(2))
    c.read(slots, k, v)
    R = R1 + R2
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    prefix = torch.zeros(2, pages_of_prompt, dtype=torch.int32, device=DEV)
    prefix[1] = 1
    q = torch.randn(R, 1, Hq, D, device=DEV, generator=g).to(torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    op = hora.GroupAttention(c, Hq, 1, torch.bfloat16, group_offsets=torch.tensor([0, R1, R], device=DEV), prefix_pages=prefix,
                             prefix_len=i32([pages_of_prompt * page, P2]), suffix_pages=i32([[2]] * R), suffix_len=i32([own] * R), status_dev=status)
    out, lse = op.run(q)
    torch.cuda.synchronize()
    assert int(status) == 0
    k, v = (x.double().repeat_interleave(Hq // Hkv, 1) for x in (k, v))     # [n, Hq, D]
    for rows, prompt, times, tol in ((slice(R1, R), slice(page, page + P2), 1, 2.0 ** -11 + 2.0 ** -10), (slice(0, R1, 50), slice(0, page), pages_of_prompt, 2.0 ** -5)):
        kk, vv = (torch.cat([x[prompt], x[2 * page:2 * page + own]]) for x in (k, v))
        z = torch.einsum("rhd,nhd->rhn", q[rows, 0].double(), kk) * D ** -0.5
        z[..., :-own] += float(torch.log(torch.tensor(float(times), dtype=torch.float64)))
        e = torch.logsumexp(z, -1)
        w = torch.exp(z - e[..., None])
        want, bound = torch.einsum("rhn,nhd->rhd", w, vv), torch.einsum("rhn,nhd->rhd", w, vv.abs())
        small = 2.0 ** -25 * kk.shape[0] * vv.abs().amax()
        assert ((out[rows, 0].double() - want).abs() <= tol * bound + 2.0 ** -8 * want.abs() + small).all()
        assert ((lse[rows, 0].double() - e).abs() <= tol).all()
