"""A prompt whose attention the contiguous forward computes, beside a cache that keeps it for the tokens after it."""
import math

import pytest
import torch

from paper_2408_10188_amd import binding as B
from paper_2408_10188_amd import paged, ring
from tests.helpers import DEV, nans

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 77, 700])
def test_a_prompt_through_the_forward_and_into_the_pages(n):
    """Q and K turned in place, the forward over them, K and V into the pages as they are: the pages hold what `append` with the rotary plan writes, bit for bit; the forward's O is
    the cache attention's, whose weights have 16 bits at least, but for its weights of 8 bits (2^-8 max |v|; both scores, off by 2 * 134 * 2^-24 of at most
    1/16 of that much each, add less than 2^-12 max |v|); and the next token sees all of it."""
    hq, hkv, d = 14, 2, 128
    gen = torch.Generator(device=DEV).manual_seed(n)
    rot = B.mmsp_rotary_plan(d, 1e6, [16, 24, 24])
    fused = torch.randn(n, hq + 2 * hkv, d, device=DEV, generator=gen).bfloat16()
    pos = torch.randint(0, 5000, (3, n), device=DEV, generator=gen, dtype=torch.int32)
    one, two = (paged.PagedCache(2, 50, 16, hq, hkv, d, 720, torch.bfloat16, DEV) for _ in range(2))
    for c in (one, two):
        c.step([c.add()], [n])
    a, b = fused.clone(), fused.clone()
    q, k, v = a[:, :hq], a[:, hq:hq + hkv], a[:, hq + hkv:]
    heads = [paged.heads_of(q), paged.heads_of(k)]
    B.mmsp_rotary_apply(rot, n, pos, n, heads, heads)
    o, lse = nans(n, hq, d), nans(hq, n)
    B.mmsp_attn_step_fwd(ring.shape_for(q, k, B.MMSP_BF16, n), B.make_block(0, n, 0, n, B.MMSP_MASK_CAUSAL_DIAG), q, k, v, o, lse, False)
    one.append(1, None, None, q, k, v)
    q2 = two.append(1, rot, pos, b[:, :hq], b[:, hq:hq + hkv], b[:, hq + hkv:])
    assert torch.equal(one.k, two.k) and torch.equal(one.v, two.v) and torch.equal(q, q2)
    o2, lse2 = nans(n, hq, d), nans(hq, n)
    two.attend(1, q2, o=o2, lse=lse2)
    assert bool(((o - o2).abs() <= (2.0 ** -8 + 2.0 ** -12) * v.float().abs().max()).all())
    assert bool(((lse - lse2).abs() <= 2.0 ** -12 * (1 + lse2.abs())).all())
    # the token after it, over both
    x = torch.randn(1, hq + 2 * hkv, d, device=DEV, generator=gen).bfloat16()
    out = []
    for c in (one, two):
        c.step(list(c.rows), [1])
        y = x.clone()
        out.append(c.attend(1, c.append(1, rot, pos[:, :1].contiguous(), y[:, :hq], y[:, hq:hq + hkv], y[:, hq + hkv:])))
    assert torch.equal(*out) and bool(torch.isfinite(out[0]).all())
