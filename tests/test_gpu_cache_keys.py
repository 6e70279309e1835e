"""Every key that a row sees is counted once, whatever the cut: with Q = 0 all weights are 1 and V says which keys were added up."""
import math

import numpy as np
import pytest
import torch

from paper_2408_10188_amd import binding as B
from paper_2408_10188_amd import paged
from tests.helpers import DEV, nans

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
CASES = [
    dict(lengths=[100003]),                                                   # one sequence over all workgroups
    dict(lengths=[65536], hq=7, hkv=1, page=128),                             # ranges that end with pages
    dict(lengths=[5003] * 16, new=[5] * 16, page=48),                         # 35 rows a KV head
    dict(lengths=[1 + 997 * i % 9000 for i in range(64)]),                    # ranges that hold several pairs
    dict(lengths=[20 + 531 * i % 3000 for i in range(200)], hq=8, hkv=8),     # more sequences than lanes
    dict(lengths=[9001, 7], new=[40, 3], hq=14, hkv=2, page=64),              # teams
    dict(lengths=[30000, 12345, 512], hq=7, hkv=1, page=16, away=0.8),        # a rank's share
    dict(lengths=[63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1023, 1024, 1025, 2047, 2048, 2049], hq=4, hkv=2),
]


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("case", CASES, ids=range(len(CASES)))
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_every_key_counts_once(case, dtype, d, order):
    """V of token j has a one at j % (d / 2) and one at d / 2 + (j / (d / 2)) % (d / 2), so O times the number of keys seen is how many of them have each remainder: whole numbers, off by
    three roundings of 2^-24 of at most 3200, far below a half, while a key that is left out, or counted twice, moves two of them by about 1."""
    lengths, new, page, hq, hkv, away = (case.get(n, x) for n, x in (("lengths", 0), ("new", None), ("page", 16), ("hq", 28), ("hkv", 4), ("away", 0.0)))
    rng, half = np.random.default_rng(5), d // 2
    used = [-(-n // page) for n in lengths]
    table = np.full((len(lengths), max(used)), -1, dtype=np.int32)
    here = (np.arange(max(used)) < np.array(used)[:, None]) & (rng.random(table.shape) >= away)
    pages = int(here.sum()) + 1
    table[here] = rng.permutation(pages)[:pages - 1]
    size = (pages, hkv, page, d) if order == "heads" else (pages, page, hkv, d)
    k, v = (torch.full(size, math.nan, dtype=dtype, device=DEV) for _ in range(2))
    if order == "tokens":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    s, j = (np.concatenate(x) for x in zip(*[(np.full(n, i), np.arange(n)) for i, n in enumerate(lengths)]))
    p = table[s, j // page].astype(np.int64)
    p, j_here = (torch.from_numpy(x[p >= 0]).to(DEV) for x in (p, j))
    k[p, :, j_here % page] = torch.randn(len(p), hkv, d, device=DEV).to(dtype)
    ones = torch.zeros(len(p), 1, d, device=DEV)
    ones.scatter_(2, (j_here % half)[:, None, None], 1.0)
    ones.scatter_(2, (half + j_here // half % half)[:, None, None], 1.0)
    v[p, :, j_here % page] = ones.expand(-1, hkv, -1).to(dtype)
    cu = None if new is None else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = len(lengths) if new is None else int(cu[-1])
    dev = [None if x is None else torch.from_numpy(np.asarray(x, dtype=np.int32)).to(DEV) for x in (table, lengths, cu)]
    q, o, lse = torch.zeros(rows, hq, d, dtype=dtype, device=DEV), nans(rows, hq, d), nans(hq, rows)
    shape = B.make_shape(hq, hkv, d, B.MMSP_F32 if dtype == F32 else B.MMSP_BF16, 1.0, (hq * d, d), (hkv * d, d), rows)
    for most_new in (0, 1 if new is None else max(new)):                       # two layouts of the same call
        cache = paged.cache_for(k, v, dev[0], dev[1], rows, dev[2], most_new)
        ws = torch.empty(B.mmsp_cache_workspace_bytes(shape, cache), dtype=torch.uint8, device=DEV)
        B.mmsp_cache_attn(shape, cache, q, None, o, lse, ws, len(ws))
        got, got_lse, row = o.double().cpu().numpy(), lse.double().cpu().numpy(), 0
        for i, n in enumerate(lengths):
            held = np.flatnonzero(np.repeat(here[i], page)[:n])
            for c in range(n - (1 if new is None else new[i]), n):
                seen = held[:np.searchsorted(held, c, side="right")]
                want = np.concatenate([np.bincount(seen % half, minlength=half), np.bincount(seen // half % half, minlength=half)])
                assert np.abs(got[row] * len(seen) - want).max() < 0.25, (i, c)
                assert (np.abs(got_lse[:, row] - math.log(len(seen))) <= 2.0 ** -20 * (1 + math.log(len(seen)))).all()
                row += 1
