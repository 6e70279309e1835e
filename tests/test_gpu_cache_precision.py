"""How exact the attention over the cache is, where its arithmetic can be seen by itself."""
import math

import numpy as np
import pytest
import torch

from paper_2408_10188_amd import binding as B
from paper_2408_10188_amd import paged
from tests.helpers import DEV, nans

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def run(q, k, v, lengths, scale, cu_new=None, page=16, seed=0):
    """k, v [seqs, hkv, tokens, d] into pages in random order; returns O in fp32 and LSE."""
    seqs, hkv, n, d = k.shape
    per = -(-n // page)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randperm(seqs * per, device=DEV, generator=gen)
    pools = []
    for x in (k, v):
        pool = torch.full((seqs * per, hkv, page, d), math.nan, dtype=x.dtype, device=DEV)
        whole = torch.full((seqs, hkv, per * page, d), math.nan, dtype=x.dtype, device=DEV)
        whole[:, :, :n] = x
        pool[ids] = whole.view(seqs, hkv, per, page, d).transpose(1, 2).reshape(seqs * per, hkv, page, d)
        pools.append(pool)
    dev = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)
    rows, hq = q.shape[:2]
    table, lengths, cu_new = ids.view(seqs, per).int(), dev(lengths), dev(cu_new)
    cache = paged.cache_for(*pools, table, lengths, rows, cu_new)
    shape = B.make_shape(hq, hkv, d, B.MMSP_F32 if q.dtype == F32 else B.MMSP_BF16, scale, (hq * d, d), (hkv * d, d), rows)
    o, lse = nans(rows, hq, d), nans(hq, rows)
    ws = torch.empty(B.mmsp_cache_workspace_bytes(shape, cache), dtype=torch.uint8, device=DEV)
    B.mmsp_cache_attn(shape, cache, q, None, o, lse, ws, len(ws))
    return o, lse


def test_weights_of_one_new_token_keep_their_bits():
    """128 keys whose V are the unit vectors: O is the weights themselves.  Head h of a KV head has Q = e_h, so a score is an element of K times 1, without error.  In units of
    2^-24 of a weight: its argument (scores in [-4, 0], up to 5.8 in base 2) is rounded as a product with log2 e, as a difference and as the difference of two wavefronts' maxima, 3 *
    5.8 ln 2 = 12; two exponentials of 2^-22, 8.  The sum's terms have the same, 20, and it is added up in 8 steps of a lane, 2 of lanes and 4 of wavefronts, 14;
    the wavefronts' results are multiplied once and added up in 4 steps, then multiplied by a reciprocal, 7.  Together 61, and 64 is 2^-18.  (Weights of 16 bits are off by up to 2^-17.)"""
    seqs, hkv, group, d = 9, 4, 7, 128
    gen = torch.Generator(device=DEV).manual_seed(1)
    k = torch.zeros(seqs, hkv, d, d, device=DEV)
    k[..., :group] = -4 * torch.rand(seqs, hkv, d, group, device=DEV, generator=gen)
    k = k.to(BF16)
    v = torch.eye(d, device=DEV, dtype=BF16).expand(seqs, hkv, d, d)
    q = torch.zeros(seqs, hkv, group, d, device=DEV, dtype=BF16)
    for h in range(group):
        q[:, :, h, h] = 1
    o, _ = run(q.view(seqs, hkv * group, d), k, v, [d] * seqs, 1.0)
    x = k[..., :group].double().cpu().numpy().transpose(0, 1, 3, 2)               # [seqs, hkv, group, keys]
    want = np.exp(x) / np.exp(x).sum(-1, keepdims=True)
    got = o.double().cpu().numpy().reshape(want.shape)
    err = np.abs(got / want - 1).max()
    assert err <= 2.0 ** -18, err


@pytest.mark.parametrize("d,hq,sums", [(64, 8, 4), (64, 40, 4), (128, 8, 4), (128, 40, 2)])
def test_scores_in_fp32_are_added_up_in_several_sums(d, hq, sums):
    """One key: LSE is the score, a sum of d products of variance 1.  Of a number x the rounding is uniform within 2^-24 |x| at most, variance x^2 / 3 in units of 2^-24.  In each of the sums, of
    m = d / sums products, the k-th rounds at variance k: m (m + 1) / 6.  Adding the sums up in pairs rounds at variances 2 m (and then, of four, 4 m).  LSE is twice a
    product of the score, d / 3 each, with log2 e (off by 0.22 units) and with ln 2 (0.05): d (2 / 3 + 0.05) together.  One sum alone, of variance
    d (d + 1) / 6, is measured at 38.8 units for d = 128 and at 19.6 for d = 64, above the bounds for four."""
    seqs, hkv = 800, 2
    gen = torch.Generator(device=DEV).manual_seed(2)
    q, k = torch.randn(seqs, hq, d, device=DEV, generator=gen), torch.randn(seqs, hkv, 1, d, device=DEV, generator=gen)
    _, lse = run(q, k, k, [1] * seqs, 1.0)
    want = (q.double().view(seqs, hkv, hq // hkv, d) * k.double()).sum(-1).view(seqs, hq).T
    rms = float((lse.double() - want).pow(2).mean().sqrt()) * 2 ** 24
    m = d / sums
    variance = sums * m * (m + 1) / 6 + (2 * 2 * m + 4 * m if sums == 4 else 2 * m) / 3 + d * (2 / 3 + 0.05)
    assert rms <= math.sqrt(variance), (rms, math.sqrt(variance))
