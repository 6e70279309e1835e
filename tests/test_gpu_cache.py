"""The paged cache on the GPU: new tokens written to it, the attention over it and the page copies, each against the fp64 oracle, and a server's
run of all of them together."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from paper_2408_10188_amd import binding as B
from paper_2408_10188_amd import paged, ring
from tests.helpers import DEV, nans, nans_like

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
THETA, SECTIONS = 1e6, {128: [16, 24, 24], 64: [8, 12, 12]}
HALF_STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


class Problem:
    """Sequences in a pool whose pages lie in random order, with NaN in every slot that no token has."""

    def __init__(self, seed, lengths, new=None, dtype=BF16, hq=28, hkv=4, d=128, page=16, order="heads", away=0.0, pad_rows=0, sigma=1.0, q_heads_extra=0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.page, self.hq, self.hkv, self.d, self.dtype, self.scale = page, hq, hkv, d, dtype, 1.0 / math.sqrt(d)
        self.lengths = np.array(lengths, dtype=np.int32)
        self.new = None if new is None else np.array(new, dtype=np.int32)
        self.cu = None if new is None else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.n_rows = (len(lengths) if new is None else int(self.cu[-1])) + pad_rows
        used = -(-np.maximum(self.lengths, 0) // page)
        width = max(1, int(used.max()) + 1)
        self.table = np.full((len(lengths), width), 10 ** 9, dtype=np.int32)   # behind a sequence: anything
        here = (np.arange(width) < used[:, None]) & (rng.random(self.table.shape) >= away)
        self.table[(np.arange(width) < used[:, None]) & ~here] = -1
        pages = int(here.sum()) + 2
        self.table[here] = rng.permutation(pages)[:int(here.sum())]
        size = (pages, hkv, page, d) if order == "heads" else (pages, page, hkv, d)
        self.k, self.v = (torch.full(size, math.nan, dtype=dtype, device=DEV) for _ in range(2))
        if order == "tokens":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        for s, n in enumerate(self.lengths):
            at = np.arange(max(n, 0))
            p, j = self.table[s, at // page].astype(np.int64), at % page
            p, j = (torch.from_numpy(x[p >= 0]).to(DEV) for x in (p, j))
            for pool in (self.k, self.v):
                pool[p, :, j] = (torch.randn(len(p), hkv, d, device=DEV, generator=gen) * sigma).to(dtype)
        self.q = (torch.randn(self.n_rows, hq + q_heads_extra, d, device=DEV, generator=gen) * sigma).to(dtype)[:, :hq]
        dev = lambda x: None if x is None else torch.from_numpy(x).to(DEV)
        self.dev = dict(page_table=dev(self.table), lengths=dev(self.lengths), cu_new=dev(self.cu))
        self.shape = ring.shape_for(self.q, self.q, B.MMSP_F32 if dtype == F32 else B.MMSP_BF16, self.n_rows, self.scale)
        self.shape.n_kv_heads = hkv
        self.cache = paged.cache_for(self.k, self.v, self.dev["page_table"], self.dev["lengths"], self.n_rows, self.dev["cu_new"])
        self.ws_bytes = B.mmsp_cache_workspace_bytes(self.shape, self.cache)
        self.ws = torch.full((self.ws_bytes + 256,), 0xff, dtype=torch.uint8, device=DEV)      # NaNs, and a guard behind it

    def run(self, stream=0):
        o_final, o, lse = nans(self.n_rows, self.hq, self.d, dtype=self.dtype), nans(self.n_rows, self.hq, self.d), nans(self.hq, self.n_rows)
        B.mmsp_cache_attn(self.shape, self.cache, self.q, o_final, o, lse, self.ws, self.ws_bytes, stream)
        assert bool((self.ws[self.ws_bytes:] == 0xff).all())
        return o_final, o, lse

    def check(self, got=None):
        """Derived bounds.  eS: an fp32 score, a sum of d products, is off by at most (d + 3) 2^-24 of the sum of their sizes; its product with log2 e and the
        subtraction of the maximum by 3 * 2^-24 of its size, and the exponential by 2^-22.  Weights are off by twice that (their sum too), by n 2^-24
        for a sum of n terms each, and in bf16 by 2^-16 more (two bf16 numbers hold 16 bits of a weight)."""
        o_final, o, lse = self.run() if got is None else got
        host = lambda t: t.double().cpu().numpy()
        want, want_lse, s_size, v_size = orc.attention(host(self.q), host(self.k), host(self.v), self.table, self.page, self.lengths, self.cu, self.scale)
        n = max(1, int(self.lengths.max()))
        e_s = (self.d + 6) * 2.0 ** -24 * s_size + 2.0 ** -22
        e_o = (2 * e_s + 2 * n * 2.0 ** -24 + (2.0 ** -16 if self.dtype == BF16 else 0.0)) * v_size
        pad = np.isnan(want_lse.T)
        for y, t, step in ((host(o), F32, 2.0 ** -22), (host(o_final), self.dtype, HALF_STEP[self.dtype] + 2.0 ** -22)):
            err, bound = np.abs(y - want), e_o[:, :, None] + step * np.abs(want)
            assert np.isnan(y[pad]).all()                                        # rows behind the last sequence: as they were
            bad = ~(err[~pad] <= bound[~pad])
            assert not bad.any(), (t, float(np.nanmax(err[~pad] / np.maximum(bound[~pad], 1e-300))))
        got_lse = host(lse).T
        assert np.isnan(got_lse[pad]).all()
        empty = ~pad & np.isneginf(want_lse.T)
        assert np.isneginf(got_lse[empty]).all() and (host(o)[empty] == 0).all() and (host(o_final)[empty] == 0).all()
        some = ~pad & ~empty
        err = np.abs(got_lse[some] - want_lse.T[some])
        assert (err <= e_s[some] + n * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(want_lse.T[some]))).all(), float(err.max())


CASES = [
    dict(lengths=[1]), dict(lengths=[16]), dict(lengths=[17]), dict(lengths=[31, 32, 33]), dict(lengths=[127, 128, 129, 130]), dict(lengths=[203], page=48),
    dict(lengths=[0, 5, 0, 700, 0]),                                              # sequences without a token: nothing is seen
    dict(lengths=[1000, 3, 517, 64, 2049], page=64, order="tokens"),
    dict(lengths=[4000], hq=7, hkv=1, page=128, away=0.6),                        # a rank's share of the pages
    dict(lengths=[300, 40], away=1.0),                                            # no page here at all
    dict(lengths=[90, 5, 260], new=[3, 0, 8], page=16),                           # ragged numbers of new tokens
    dict(lengths=[90, 5, 260], new=[90, 2, 31], page=48, pad_rows=5, order="tokens"),   # a whole short prompt, rows behind the last sequence
    dict(lengths=[3, 40], new=[7, 40], hq=4, hkv=2),                              # more rows than tokens: the first see nothing
    dict(lengths=[1500, 900], new=[5, 1], hq=8, hkv=8, page=32, q_heads_extra=3), # no grouping, Q inside a wider projection
    dict(lengths=[777], new=[16], hq=40, hkv=2, page=16),                         # groups of 20 heads
    dict(lengths=[5, 600, 33], hq=64, hkv=2),                                     # 32 heads a group, one token
    dict(lengths=[5, 1, 1, 1, 1, 1, 1, 1] * 40, hq=4, hkv=2),                     # many short sequences
    dict(lengths=list(range(1, 600, 7)), hq=2, hkv=1, new=[1 + i % 2 if i else 1 for i in range(86)]),
    dict(lengths=[64 * 300 + 5], hq=7, hkv=1, page=16, sigma=2.0),                # many partial results, sharper weights
]


@pytest.mark.parametrize("case", CASES, ids=range(len(CASES)))
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 128), (F32, 64)])
def test_attention_over_the_cache(case, dtype, d):
    Problem(len(case["lengths"]), dtype=dtype, d=d, **case).check()


def test_repeats_bit_for_bit_and_on_other_streams():
    p = Problem(5, [1, 3000, 40, 9000], page=16)
    first = p.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = p.run(s.cuda_stream)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("which", [(True, False, False), (False, True, False), (False, False, True), (True, False, True)])
def test_any_of_the_results(which):
    p = Problem(6, [700, 20])
    full = p.run()
    out = [nans_like(t) if w else None for t, w in zip(full, which)]
    B.mmsp_cache_attn(p.shape, p.cache, p.q, out[0], out[1], out[2], p.ws, p.ws_bytes)
    assert all(torch.equal(a, b) for a, b in zip(full, out) if b is not None)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_has_no_influence(dtype, value):
    """K and V of the later of five new tokens hold infinities or NaN: the rows before them are as without, bit for bit."""
    lengths, new, d = [77, 150], [5, 5], 128
    p = Problem(7, lengths, new, dtype=dtype, hq=14, hkv=2, page=16)
    clean = p.run()
    for s, n in enumerate(lengths):
        page, slot = int(p.table[s, (n - 2) // 16]), (n - 2) % 16
        p.k[page, 0, slot, 3] = value
        p.v[page, :, slot, ::3] = value
    odd = p.run()
    before = torch.tensor([0, 1, 2, 5, 6, 7], device=DEV)
    for a, b in zip(clean, odd):
        a, b = (a, b) if a.shape[0] == 10 else (a.T, b.T)
        assert torch.equal(a[before], b[before])
    after = odd[1][torch.tensor([3, 4, 8, 9], device=DEV)]
    assert not bool(torch.isfinite(after[:, :, ::3]).any())
    if math.isnan(value):                                   # a NaN among the scores: the row's LSE and all of its O
        assert bool(torch.isnan(after[:, :7]).all()) and bool(torch.isnan(odd[2][:7, 3]).all())
    assert bool(torch.isfinite(after[:, 7:, 1::3]).all())


def test_scores_of_minus_infinity_are_like_nothing_seen():
    p = Problem(8, [40], hq=2, hkv=1, dtype=F32, d=64)
    p.q.fill_(1.0)
    p.k[:, :, :, 0] = -math.inf
    p.k[:, :, :, 1:] = 0.0
    o_final, o, lse = p.run()
    assert bool((o == 0).all()) and bool((o_final == 0).all()) and bool((lse == -math.inf).all())


def test_ids_and_lengths_that_are_out_of_range():
    """Pages beyond the pool are not here, a length beyond the table counts as the table's, a negative one as none."""
    p = Problem(9, [100, 64, 48], page=16, hq=4, hkv=2)
    want = p.run()
    p.dev["page_table"][0, 1], p.dev["page_table"][0, 2] = p.k.shape[0], -2 ** 31
    p.table[0, 1:3] = -1
    p.check()
    wide = p.dev["page_table"][:, :3].contiguous()         # 48 tokens at most
    p.dev["lengths"][:] = torch.tensor([48, 2 ** 31 - 1, -5], dtype=torch.int32)
    p.cache = paged.cache_for(p.k, p.v, wide, p.dev["lengths"], 3)
    p.table, p.lengths = p.table[:, :3], np.array([48, 48, 0], dtype=np.int32)
    p.check()
    assert not torch.equal(want[0], p.run()[0])


def test_partial_results_of_ranks_are_joined_by_merge():
    """Each rank holds the pages that the others do not; log-sum-exp merges of their (O, LSE) are the whole."""
    whole = Problem(10, [3000, 77, 16], page=16)
    want = whole.run()
    o_acc, lse_acc = torch.zeros_like(want[1]), torch.full_like(want[2], -math.inf)
    out = nans_like(want[0])
    for rank in range(3):
        table = whole.dev["page_table"].clone()
        table[:, torch.arange(table.shape[1], device=DEV) % 3 != rank] = -1
        cache = paged.cache_for(whole.k, whole.v, table, whole.dev["lengths"], 3)
        o, lse = nans_like(want[1]), nans_like(want[2])
        B.mmsp_cache_attn(whole.shape, cache, whole.q, None, o, lse, whole.ws, whole.ws_bytes)
        B.mmsp_attn_merge(whole.shape, 0, 3, o_acc, lse_acc, o, lse, out if rank == 2 else None)
    whole.check((out, o_acc, lse_acc))


def test_long_pool_and_far_offsets():
    """A pool of more than 2^31 elements: pages near its end are read and written where they lie."""
    pages, page, hkv, d = 2 ** 31 // (4 * 64 * 128) + 40, 64, 4, 128
    k, v = (torch.empty(pages, hkv, page, d, dtype=BF16, device=DEV) for _ in range(2))
    gen = torch.Generator(device=DEV).manual_seed(2)
    small = [torch.randn(4, hkv, page, d, device=DEV, generator=gen).bfloat16() for _ in range(2)]
    ids = [pages - 1, 3, pages - 20, 0]
    q = torch.randn(1, 28, d, device=DEV, generator=gen).bfloat16()
    for i, p in enumerate(ids):
        k[p], v[p] = small[0][i], small[1][i]
    new_k, new_v = (torch.randn(1, hkv, d, device=DEV, generator=gen).bfloat16() for _ in range(2))
    got = []
    for kk, vv, table in ((k, v, ids), (*small, [0, 1, 2, 3])):
        table = torch.tensor([table], dtype=torch.int32, device=DEV)
        lengths = torch.tensor([3 * 64 - 5], dtype=torch.int32, device=DEV)
        shape, cache = ring.shape_for(q, new_k, B.MMSP_BF16, 1), paged.cache_for(kk, vv, table, lengths, 1)
        B.mmsp_cache_append(shape, cache, None, None, 0, None, new_k, new_v)
        o, ws = nans_like(q), torch.empty(B.mmsp_cache_workspace_bytes(shape, cache), dtype=torch.uint8, device=DEV)
        B.mmsp_cache_attn(shape, cache, q, o, None, None, ws, len(ws))
        page_2 = kk[int(table[0, 2])].clone()
        copies = torch.tensor([[int(table[0, 2]), int(table[0, 3]), 64]], dtype=torch.int32, device=DEV)
        B.mmsp_cache_copy_pages(paged.shape_for(kk, B.MMSP_BF16), cache, 1, 0, copies, 1)
        got.append((o, page_2, kk[int(table[0, 3])].clone()))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and torch.equal(got[0][1], got[0][2])
    assert torch.equal(got[0][1][:, 64 - 6], new_k[0])


# ---- append ----

@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("case", [dict(lengths=[5]), dict(lengths=[1, 16, 17, 300], page=16, order="tokens"), dict(lengths=[200, 7, 90], new=[150, 0, 3], page=48, pad_rows=4),
                                  dict(lengths=[3, 50], new=[9, 2], hq=4, hkv=2), dict(lengths=[500, 60], new=[400, 60], away=0.5, hq=8, hkv=8)], ids=range(5))
@pytest.mark.parametrize("turned", [True, False])
def test_append(case, dtype, d, turned):
    p = Problem(11, dtype=dtype, d=d, q_heads_extra=2 * case.get("hkv", 4) + 1, **case)
    gen = torch.Generator(device=DEV).manual_seed(12)
    k, v = (torch.randn(p.n_rows, 3 * p.hkv, d, device=DEV, generator=gen).to(dtype)[:, p.hkv:2 * p.hkv] for _ in range(2))
    pos = torch.randint(0, 1 << 18, (3, p.n_rows + 2), device=DEV, generator=gen, dtype=torch.int32)
    before = p.k.clone(), p.v.clone(), p.q.clone()
    room = nans(p.n_rows + 3, p.hq, d, dtype=dtype)        # q_out is dense, Q lies in wider rows; a guard behind it
    q_out = room[:p.n_rows]
    shape = B.make_shape(p.hq, p.hkv, d, B.MMSP_F32 if dtype == F32 else B.MMSP_BF16, 1.0, (p.q.stride(0), d), (k.stride(0), d), p.n_rows)
    rot = B.mmsp_rotary_plan(d, THETA, SECTIONS[d]) if turned else None
    B.mmsp_cache_append(shape, p.cache, rot, pos, pos.stride(0), p.q, k, v, q_out)
    want_q, want_k = p.q.clone(), k.clone()
    if turned:                                              # the standalone call's arithmetic, bit for bit (it is tested against the oracle)
        x, y = [p.q, k.contiguous()], [torch.empty(p.n_rows, p.hq, d, dtype=dtype, device=DEV), torch.empty(p.n_rows, p.hkv, d, dtype=dtype, device=DEV)]
        B.mmsp_rotary_apply(rot, p.n_rows, pos, pos.stride(0), [paged.heads_of(t) for t in x], [paged.heads_of(t) for t in y])
        want_q, want_k = y
    rows = p.n_rows if p.cu is None else int(p.cu[-1])
    assert torch.equal(q_out[:rows], want_q[:rows]) and bool(torch.isnan(room[rows:]).all()) and torch.equal(p.q, before[2])
    host = [t.float().cpu().numpy() for t in (*before[:2], want_k, v)]
    orc.append(host[0], host[1], p.table, p.page, p.lengths, p.cu, host[2], host[3])
    for got, want in zip((p.k, p.v), host[:2]):             # every other slot as it was, NaN in the unused ones
        assert np.array_equal(got.float().cpu().numpy(), want, equal_nan=True)
    # Q in place
    B.mmsp_cache_append(shape, p.cache, rot, pos, pos.stride(0), p.q, k, v, p.q)
    assert torch.equal(p.q[:rows], want_q[:rows]) and torch.equal(p.q[rows:], before[2][rows:])


# ---- page copies ----

@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("hkv,page,layers", [(4, 16, 3), (1, 48, 1), (3, 256, 2)])
def test_page_copies(dtype, d, order, hkv, page, layers):
    n_pages = 30
    rng = np.random.default_rng(page)
    pool = lambda: torch.randn(layers, n_pages, *((hkv, page) if order == "heads" else (page, hkv)), d, device=DEV).to(dtype)
    k, v = (x if order == "heads" else x.transpose(2, 3) for x in (pool(), pool()))
    ids = rng.permutation(n_pages)
    copies = np.stack([ids[:9][rng.integers(0, 4, 9)], ids[9:18], rng.integers(1, page + 1, 9)], 1).astype(np.int32)
    copies[0, 2], copies[1, 2], copies[2, 2] = page, 1, page + 1000             # more than a page counts as one
    odd = np.array([[-1, ids[20], page], [n_pages, ids[21], page], [ids[0], -1, page], [ids[0], n_pages, 3], [ids[22], ids[22], page], [ids[0], ids[23], 0], [ids[0], ids[24], -7]],
                   dtype=np.int32)                                              # nothing of these is done
    want = [x.clone() for x in (k, v)]
    for s, t, n in copies.tolist():
        for x in want:
            x[:, t, :, :n] = x[:, s, :, :n]
    dev = torch.from_numpy(np.concatenate([copies[:4], odd, copies[4:]])).to(DEV)
    B.mmsp_cache_copy_pages(paged.shape_for(k[0], B.MMSP_F32 if dtype == F32 else B.MMSP_BF16), paged.cache_for(k[0], v[0]), layers, k.stride(0), dev, len(dev))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


# ---- a captured step ----

def test_a_captured_step_follows_its_arrays():
    """Append and attention captured once; between the replays the lengths, the tables, the tokens and the positions change, with eager work beside."""
    p = Problem(13, [30, 500, 7], page=16)
    d, hkv = p.d, p.hkv
    width = 40
    table = torch.full((3, width), -1, dtype=torch.int32, device=DEV)
    k_pool, v_pool = (torch.randn(120, hkv, 16, d, device=DEV).bfloat16() for _ in range(2))
    table[:] = torch.arange(120, device=DEV).view(3, width)
    lengths = torch.tensor([30, 500, 7], dtype=torch.int32, device=DEV)
    q, k, v = (torch.randn(3, h, d, device=DEV).bfloat16() for h in (28, hkv, hkv))
    pos = torch.zeros(3, 3, dtype=torch.int32, device=DEV)
    shape, cache, rot = ring.shape_for(q, k, B.MMSP_BF16, 3), paged.cache_for(k_pool, v_pool, table, lengths, 3), B.mmsp_rotary_plan(d, THETA, SECTIONS[d])
    ws = torch.empty(B.mmsp_cache_workspace_bytes(shape, cache), dtype=torch.uint8, device=DEV)
    eager_ws = torch.empty_like(ws)
    out = [nans_like(q), nans(3, 28, d), nans(28, 3), nans_like(q)]

    def step(o, w, stream):
        B.mmsp_cache_append(shape, cache, rot, pos, 3, q, k, v, o[3], stream)
        B.mmsp_cache_attn(shape, cache, o[3], o[0], o[1], o[2], w, len(w), stream)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(out, ws, torch.cuda.current_stream().cuda_stream)
    rng = np.random.default_rng(3)
    for i in range(5):
        new = torch.from_numpy(rng.integers(1, 640, 3).astype(np.int32)).to(DEV)
        lengths.copy_(new)
        pos.copy_(torch.from_numpy(rng.integers(0, 1 << 17, (3, 3)).astype(np.int32)))
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device=DEV))
        table.copy_(table.view(-1)[torch.randperm(120, device=DEV)].view(3, width))
        pools = k_pool.clone(), v_pool.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, wrote = [t.clone() for t in out], (k_pool.clone(), v_pool.clone())
        k_pool.copy_(pools[0])
        v_pool.copy_(pools[1])
        mine = [nans_like(t) for t in out]
        step(mine, eager_ws, 0)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, mine)) and torch.equal(wrote[0], k_pool) and torch.equal(wrote[1], v_pool)


# ---- a server's run ----

def test_a_server_run():
    """Two layers: a video's prompt, three continuations forked from it, steps of one and of a few tokens, one freed, the pool compacted, and on; each
    attention against the oracle over everything that its sequence was given."""
    layers, hq, hkv, d, page = 2, 14, 2, 128, 16
    cache = paged.PagedCache(layers, 36, page, hq, hkv, d, 400, BF16, DEV)
    rot = B.mmsp_rotary_plan(d, THETA, SECTIONS[d])
    gen = torch.Generator(device=DEV).manual_seed(4)
    given = {}                                              # sequence -> per layer (K turned, V), host fp64

    def run(seqs, n_new):
        cache.step(seqs, n_new)
        n = sum(n_new)
        if n == 0:
            return
        pos = torch.randint(0, 5000, (3, n), device=DEV, generator=gen, dtype=torch.int32)
        for layer in range(layers):
            x = torch.randn(n, hq + 2 * hkv, d, device=DEV, generator=gen).bfloat16()
            q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
            k_turned = torch.empty(n, hkv, d, dtype=BF16, device=DEV)
            B.mmsp_rotary_apply(rot, n, pos, n, [paged.heads_of(k)], [paged.heads_of(k_turned)])
            q = cache.append(layer, rot, pos, q, k, v)
            o = cache.attend(layer, q)
            row = 0
            for s, m in zip(seqs, n_new):
                kk, vv = (t[row:row + m].double().cpu().numpy() for t in (k_turned, v))
                old = given.setdefault(s, [(np.zeros((0, hkv, d)),) * 2] * layers)
                given[s] = [tuple(np.concatenate(x) for x in zip(old[i], (kk, vv))) if i == layer else old[i] for i in range(layers)]
                if m == 0:
                    continue
                K, V = given[s][layer]
                total = len(K)
                want, _, s_size, v_size = orc.attention(q[row:row + m].double().cpu().numpy(), K.transpose(1, 0, 2)[None], V.transpose(1, 0, 2)[None], [[0]], total, [total],
                                                        [0, m], 1 / math.sqrt(d))
                bound = ((2 * (d + 6) * s_size + 2 * total) * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -16)[:, :, None] * v_size[:, :, None] + (2.0 ** -8 + 2.0 ** -22) * np.abs(want)
                assert (np.abs(o[row:row + m].double().cpu().numpy() - want) <= bound).all()
                row += m
    a = cache.add()
    run([a], [150])
    forks = [cache.fork(a) for _ in range(3)]
    for s in forks:
        given[s] = list(given[a])
    run([a, *forks], [1, 1, 1, 1])                          # the last page, half full, becomes everybody's own
    run([forks[2], forks[0]], [20, 3])
    cache.free(a)
    used = int((cache._refs > 0).sum())
    assert cache.compact() == used
    run([forks[0], forks[1], forks[2]], [4, 0, 1])
    b = cache.add()
    run([b, forks[1]], [33, 1])
    state = cache._refs.copy(), {s: r.copy() for s, r in cache.rows.items()}
    with pytest.raises(B.MmspError) as e:                   # the last one has no room: nothing is taken, shared pages stay shared
        extra = cache.fork(forks[1])
        state = cache._refs.copy(), {s: r.copy() for s, r in cache.rows.items()}
        cache.step([extra, b, forks[1]], [2, 100, 240])
    assert e.value.status == B.MMSP_ERR_NO_PAGES
    assert np.array_equal(state[0], cache._refs) and all(np.array_equal(r, cache.rows[s]) for s, r in state[1].items())
    assert cache.pages.n_free == int((cache._refs == 0).sum()) and set(cache._free[:cache.pages.n_free]) == set(np.flatnonzero(cache._refs == 0))
    given[extra] = list(given[forks[1]])
    run([forks[1], extra], [1, 5])
