"""The paged cache's calls at the ends of their ranges: page tables far wider than the sequences, more sequences than a workgroup's threads, rows in several
groups with something in the keys that only the later ones see, and more rows than a grid has workgroups."""
import math

import pytest
import torch

from paper_2408_10188_amd import binding as B
from paper_2408_10188_amd import paged
from tests.helpers import DEV
from tests.test_gpu_cache import BF16, F32, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("case", [dict(lengths=[1]), dict(lengths=[5, 0, 40]), dict(lengths=list(range(100)), hq=4, hkv=2), dict(lengths=[16, 2100], new=[2, 3]),
                                  dict(lengths=[3 + 37 * i % 90 for i in range(1500)] + [3000], new=[i % 3 for i in range(1501)], hq=2, hkv=1, pad_rows=2)], ids=range(5))
def test_tables_wider_than_the_sequences(case, dtype, d):
    """Room for 64 thousand tokens each, as a server's table has: the layout of the call follows the room, its work the lengths."""
    p = Problem(21, dtype=dtype, d=d, **case)
    wide = torch.full((len(p.lengths), 4096), 10 ** 9, dtype=torch.int32, device=DEV)
    wide[:, :p.table.shape[1]] = p.dev["page_table"]
    p.cache = paged.cache_for(p.k, p.v, wide, p.dev["lengths"], p.n_rows, p.dev["cu_new"])
    p.ws_bytes = B.mmsp_cache_workspace_bytes(p.shape, p.cache)
    p.ws = torch.full((p.ws_bytes + 256,), 0xff, dtype=torch.uint8, device=DEV)
    p.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_groups_of_rows_that_do_not_see_the_same(dtype, value):
    """40 new tokens of 7 heads a KV head, 280 rows in 9 groups: those before the odd token are as without it, bit for bit."""
    p = Problem(22, [70, 700], [40, 40], dtype=dtype, hq=14, hkv=2, page=32)
    clean = p.run()
    for s, n in enumerate((70, 700)):
        token = n - 40 + 23
        page, slot = int(p.table[s, token // 32]), token % 32
        p.k[page, 0, slot, 5] = value
        p.v[page, :, slot, 1::2] = value
    odd = p.run()
    sees = torch.tensor([i % 40 >= 23 for i in range(80)], device=DEV)
    for a, b in zip(clean, odd):
        a, b = (a, b) if a.shape[0] == 80 else (a.T, b.T)
        assert torch.equal(a[~sees], b[~sees])
    assert not bool(torch.isfinite(odd[1][sees][:, :, 1::2]).any())
    assert bool(torch.isfinite(odd[1][sees][:, 7:, ::2]).all())


def test_more_rows_than_a_grid_has_workgroups():
    """2^24 rows, of which the last few of each sequence have tokens that exist.  (The rows overlap in memory; they are only read.)"""
    hkv, d, page = 17, 64, 16
    new = [(1 << 24) - 1, 4]
    rows, lengths = sum(new), [5, 3]
    k, v = (torch.rand((rows + hkv) * d, device=DEV) for _ in range(2))
    kp, vp = (torch.full((2, hkv, page, d), math.nan, device=DEV) for _ in range(2))
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    cache = paged.cache_for(kp, vp, dev([[1], [0]]), dev(lengths), rows, dev([0, new[0], rows]))
    shape = B.make_shape(hkv, hkv, d, B.MMSP_F32, 1.0, (d, d), (d, d), 0)
    B.mmsp_cache_append(shape, cache, None, None, 0, None, k, v)
    want = [torch.full_like(kp, math.nan) for _ in range(2)]
    for t, (s, n) in enumerate(zip((1, 0), lengths)):
        last = (new[0], rows)[t]
        for j in range(n):
            at = (last - n + j) * d
            for w, x in zip(want, (k, v)):
                w[s, :, j] = x[at:at + hkv * d].view(hkv, d)
    for got, w in zip((kp, vp), want):
        assert torch.equal(got.nan_to_num(-1.0), w.nan_to_num(-1.0))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [[2], [4, 4], [5, 5], [6], [7, 7], [13], [14, 14], [20], [21], [28, 28], [54], [55], [110], [1, 20, 0, 6], [0, 0, 9], [40, 1, 1, 1, 1]],
                         ids=lambda x: "-".join(map(str, x)))
def test_numbers_of_rows_around_the_layouts(new, dtype):
    """Seven heads a KV head: 14 to 770 rows, one group, teams of two, four and eight, full and not, and more groups than a team takes at once; with the
    same number of new tokens in every sequence and with ragged ones."""
    lengths = [n + 100 + 517 * (i % 3) for i, n in enumerate(new)]
    Problem(23, lengths, new, dtype=dtype, hq=14, hkv=2, page=16, pad_rows=len(new) % 2).check()
    Problem(24, [n + 3000 for n in new], new, dtype=dtype, hq=7, hkv=1, page=64).check()


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("lengths", [[5003] * 16, [100 + 9 * i * i % 2900 for i in range(33)], [30 + 1291 * i % 4000 for i in range(64)]], ids=["even", "33", "64"])
def test_cuts_of_batches(lengths, dtype, d):
    """Ranges of several tiles for one workgroup a CU, one tile for each of two, and pairs of very different lengths in a range."""
    Problem(25, lengths, dtype=dtype, d=d, hq=8, hkv=4, page=64).check()


@pytest.mark.parametrize("first", [0, 4])
def test_rows_before_the_first_sequence(first):
    """The rows of a call may begin anywhere: what lies before cu_new[0] and behind cu_new[n_seqs] is left alone, by the joining launch too."""
    whole = Problem(26, [4000, 3, 900], [3, 1, 2], hq=14, hkv=2, page=64, pad_rows=7)
    want = whole.run()
    q = torch.roll(whole.q, first, 0).contiguous()
    cu = whole.dev["cu_new"] + first
    cache = paged.cache_for(whole.k, whole.v, whole.dev["page_table"], whole.dev["lengths"], whole.n_rows, cu)
    got = [torch.full_like(t, math.nan) for t in want]
    B.mmsp_cache_attn(whole.shape, cache, q, *got, whole.ws, whole.ws_bytes)
    for a, b in zip(want, got):
        a, b = (a, b) if a.shape[0] == whole.n_rows else (a.T, b.T)
        assert torch.equal(a[:6], b[first:first + 6])
        assert bool(torch.isnan(b[:first]).all()) and bool(torch.isnan(b[first + 6:]).all())


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
def test_new_tokens_behind_the_tables_end(dtype, d):
    """Lengths that have gone past the page tables (48 tokens), by one, by a few, as far as an int32 goes: those tokens are nowhere.  None of the tokens that are there is
    written over, and the new ones before the end keep their numbers, in the append and in the attention."""
    page, hkv, room = 16, 2, 48
    lengths, new = [49, 50, 48, 2 ** 31 - 1, 60], [1, 4, 2, 5, 12]
    cu = [0, 1, 5, 7, 12, 24]
    gen = torch.Generator(device=DEV).manual_seed(3)
    k_pool, v_pool = (torch.randn(15, hkv, page, d, device=DEV, generator=gen).to(dtype) for _ in range(2))
    q, k, v = (torch.randn(cu[-1], h, d, device=DEV, generator=gen).to(dtype) for h in (4, hkv, hkv))
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    table, seen = torch.arange(15, device=DEV, dtype=torch.int32).view(5, 3), dev(lengths)
    for per_seq in (True, False):                           # one new token each, then the ragged numbers
        n_rows = 5 if per_seq else cu[-1]
        starts = None if per_seq else dev(cu)
        cache = paged.cache_for(k_pool, v_pool, table, seen, n_rows, starts)
        shape = B.make_shape(4, hkv, d, B.MMSP_F32 if dtype == F32 else B.MMSP_BF16, 0.1, (4 * d, d), (hkv * d, d), n_rows)
        rows = [(s, s, lengths[s] - 1) for s in range(5)] if per_seq else [(cu[s] + i, s, lengths[s] - new[s] + i) for s in range(5) for i in range(new[s])]
        want = k_pool.clone(), v_pool.clone()
        for r, s, token in rows:
            if token < room:
                for pool, x in zip(want, (k, v)):
                    pool[3 * s + token // page, :, token % page] = x[r]
        B.mmsp_cache_append(shape, cache, None, None, 0, None, k, v)
        assert torch.equal(k_pool, want[0]) and torch.equal(v_pool, want[1])
        # what each row sees, as sequences of their own whose only new token is the row
        o, lse = torch.full((n_rows, 4, d), math.nan, device=DEV), torch.full((4, n_rows), math.nan, device=DEV)
        ws = torch.empty(B.mmsp_cache_workspace_bytes(shape, cache), dtype=torch.uint8, device=DEV)
        B.mmsp_cache_attn(shape, cache, q, None, o, lse, ws, len(ws))
        alone_table, alone = table[torch.tensor([s for _, s, _ in rows], device=DEV)].contiguous(), dev([min(token + 1, room) for _, _, token in rows])
        shape = B.make_shape(4, hkv, d, shape.io_dtype, 0.1, (4 * d, d), (hkv * d, d), n_rows)
        cache = paged.cache_for(k_pool, v_pool, alone_table, alone, n_rows)
        want_o, want_lse = torch.full_like(o, math.nan), torch.full_like(lse, math.nan)
        ws = torch.empty(B.mmsp_cache_workspace_bytes(shape, cache), dtype=torch.uint8, device=DEV)
        B.mmsp_cache_attn(shape, cache, q, None, want_o, want_lse, ws, len(ws))
        # both sum at most 48 terms in fp32, weights with 16 bits at least: a row that sees a key more or less is off by far more (a weight of 1/48 or so)
        assert bool(((o - want_o).abs() <= 1e-4).all()) and bool(((lse - want_lse).abs() <= 1e-5).all())
