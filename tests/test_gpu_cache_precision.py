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
