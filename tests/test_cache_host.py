"""CPU side of the inference calls: the rotary plan, page bookkeeping against a plain model of it, and the refusals of every call (nothing
here launches a kernel)."""
import math
import random

import numpy as np
import pytest

from oracle import paged_oracle as orc
from paper_2408_10188_amd import binding as B

FAKE = 0x1000


# ---- rotary plan ----

@pytest.mark.parametrize("d,theta,sections", [(128, 1e6, [16, 24, 24]), (64, 1e4, [32]), (128, 1.0, [64]), (128, 1e6, [0, 64, 0, 0]), (64, 5e5, [1, 31])])
def test_rotary_plan(d, theta, sections):
    r = B.mmsp_rotary_plan(d, theta, sections)
    assert (r.head_dim, r.n_axes) == (d, len(sections))
    assert list(r.axis)[:d // 2] == [a for a, n in enumerate(sections) for _ in range(n)]
    for i in range(d // 2):
        want = theta ** (-2.0 * i / d) / (2 * math.pi)
        # pow and the product with 1 / (2 pi) are off by a few units in the 53rd bit each
        assert abs(r.turns[i] / 2.0 ** 64 - want) <= 8 * 2.0 ** -53 * want + 2.0 ** -64


@pytest.mark.parametrize("args,status", [((96, 1e6, [48]), B.MMSP_ERR_UNSUPPORTED), ((128, 0.5, [64]), B.MMSP_ERR_INVALID_ARG),
                                         ((128, math.nan, [64]), B.MMSP_ERR_INVALID_ARG), ((128, math.inf, [64]), B.MMSP_ERR_INVALID_ARG),
                                         ((128, 1e6, [63]), B.MMSP_ERR_INVALID_ARG), ((128, 1e6, [65, -1]), B.MMSP_ERR_INVALID_ARG),
                                         ((128, 1e6, []), B.MMSP_ERR_INVALID_ARG), ((128, 1e6, [16, 16, 16, 8, 8]), B.MMSP_ERR_INVALID_ARG)])
def test_rotary_plan_refuses(args, status):
    with pytest.raises(B.MmspError) as e:
        B.mmsp_rotary_plan(*args)
    assert e.value.status == status and str(e.value)


def _refused(status, f, *args):
    with pytest.raises(B.MmspError) as e:
        f(*args)
    assert e.value.status == status, str(e.value)


def test_rotary_apply_refuses():
    rot = B.mmsp_rotary_plan(128, 1e6, [16, 24, 24])
    bad = B.MMSP_ERR_INVALID_ARG
    h = lambda data=FAKE, n=4, dtype=B.MMSP_BF16, ts=512, hs=128: B.make_heads(data, n, dtype, ts, hs)
    call = lambda rows=5, pos=FAKE, stride=5, x=(h(),), y=(h(2 * FAKE),), r=rot: (r, rows, pos, stride, list(x), list(y))
    for args in (call(rows=-1), call(rows=(1 << 26) + 1, stride=1 << 27), call(pos=None), call(stride=4), call(x=(h(None),)), call(x=(h(FAKE + 8),)),
                 call(x=(h(n=0),)), call(x=(h(n=3),)), call(x=(h(dtype=2),)), call(x=(h(ts=120),)), call(x=(h(ts=516),)), call(y=(h(hs=64),)),
                 call(x=(h(), h(dtype=B.MMSP_F32)), y=(h(2 * FAKE), h(3 * FAKE, dtype=B.MMSP_F32))), call(x=(), y=()), call(x=(h(),) * 3, y=(h(),) * 3),
                 call(y=(h(ts=1024),)), call(x=(h(dtype=B.MMSP_F32),), y=(h(),))):            # the last two: in place with other strides, another type
        _refused(bad, B.mmsp_rotary_apply, *args)
    _refused(B.MMSP_ERR_UNSUPPORTED, B.mmsp_rotary_apply, *call(y=(h(2 * FAKE, dtype=B.MMSP_F32),)))
    other = B.mmsp_rotary_plan(128, 1e6, [64])
    other.axis[7] = 1                                                                          # an axis that there is not
    _refused(bad, B.mmsp_rotary_apply, *call(r=other))
    other = B.mmsp_rotary_plan(128, 1e6, [64])
    other.head_dim = 256
    _refused(B.MMSP_ERR_UNSUPPORTED, B.mmsp_rotary_apply, *call(r=other))


# ---- calls on the cache ----

def _shape(**kw):
    base = dict(n_q_heads=4, n_kv_heads=2, head_dim=128, io_dtype=B.MMSP_BF16, softmax_scale=0.1, q_strides=(512, 128), kv_strides=(256, 128), lse_head_stride=3)
    return B.make_shape(**{**base, **kw})


def _cache(**kw):
    base = dict(k=FAKE, v=FAKE, strides=(4096, 128, 2048), n_pages=9, page_size=16, page_table=FAKE, table_stride=4, max_pages=4, n_seqs=3, lengths=FAKE,
                cu_new=None, n_rows=3)
    return B.make_cache(**{**base, **kw})


@pytest.mark.parametrize("kw", [dict(n_pages=-1), dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(page_size=0), dict(page_size=24), dict(page_size=-16),
                                dict(strides=(64, 128, 2048)), dict(strides=(4096, 64, 2048)), dict(strides=(4096, 128, 2044)),
                                dict(strides=(4096, (1 << 23) + 8, 2048)), dict(max_pages=0), dict(max_pages=1 << 27, table_stride=1 << 27),
                                dict(n_seqs=-1, n_rows=-1), dict(n_rows=2), dict(n_rows=(1 << 26) + 1, cu_new=FAKE), dict(page_table=None),
                                dict(lengths=None), dict(table_stride=3)])
def test_cache_calls_refuse_bad_caches(kw):
    cache, shape = _cache(**kw), _shape()
    _refused(B.MMSP_ERR_INVALID_ARG, B.mmsp_cache_append, shape, cache, None, None, 0, FAKE, FAKE, FAKE, FAKE)
    _refused(B.MMSP_ERR_INVALID_ARG, B.mmsp_cache_attn, shape, cache, FAKE, FAKE, None, None, FAKE, 1 << 40)
    assert B.mmsp_cache_workspace_bytes(shape, cache) == 0


def test_cache_calls_refuse_bad_arguments():
    shape, cache, bad = _shape(), _cache(), B.MMSP_ERR_INVALID_ARG
    rot = B.mmsp_rotary_plan(128, 1e6, [16, 24, 24])
    _refused(bad, B.mmsp_cache_append, shape, cache, rot, None, 3, FAKE, FAKE, FAKE, FAKE)             # no positions
    _refused(bad, B.mmsp_cache_append, shape, cache, rot, FAKE, 2, FAKE, FAKE, FAKE, FAKE)             # axes overlap
    _refused(bad, B.mmsp_cache_append, shape, cache, B.mmsp_rotary_plan(64, 1e6, [32]), FAKE, 3, FAKE, FAKE, FAKE, FAKE)
    _refused(bad, B.mmsp_cache_append, shape, cache, None, None, 0, None, FAKE, FAKE, FAKE)            # q_out without q
    _refused(bad, B.mmsp_cache_append, shape, cache, None, None, 0, FAKE, None, FAKE, FAKE)
    _refused(bad, B.mmsp_cache_append, shape, cache, None, None, 0, FAKE, FAKE, FAKE + 4, FAKE)
    _refused(bad, B.mmsp_cache_attn, shape, cache, None, FAKE, None, None, FAKE, 1 << 40)
    _refused(bad, B.mmsp_cache_attn, shape, cache, FAKE, None, None, None, FAKE, 1 << 40)              # no result
    _refused(bad, B.mmsp_cache_attn, shape, cache, FAKE, FAKE + 4, None, None, FAKE, 1 << 40)
    _refused(bad, B.mmsp_cache_attn, _shape(lse_head_stride=2), cache, FAKE, FAKE, None, FAKE, FAKE, 1 << 40)
    _refused(bad, B.mmsp_cache_attn, shape, cache, FAKE, FAKE, None, None, FAKE + 4, 1 << 40)
    need = B.mmsp_cache_workspace_bytes(shape, cache)
    assert need > 0
    for ws, nbytes in ((None, need), (FAKE, need - 1)):
        _refused(B.MMSP_ERR_WORKSPACE_TOO_SMALL, B.mmsp_cache_attn, shape, cache, FAKE, FAKE, None, None, ws, nbytes)
    _refused(B.MMSP_ERR_UNSUPPORTED, B.mmsp_cache_attn, shape, _cache(n_rows=(1 << 21) + 1, cu_new=FAKE), FAKE, FAKE, None, None, FAKE, 1 << 40)
    _refused(B.MMSP_ERR_UNSUPPORTED, B.mmsp_cache_attn, _shape(head_dim=64), cache, FAKE, FAKE, None, None, FAKE, 1 << 40)
    for kw in (dict(n_layers=-1), dict(n_copies=-1), dict(layer_stride=4), dict(copies=None)):
        a = {**dict(n_layers=2, layer_stride=4096 * 9, copies=FAKE, n_copies=1), **kw}
        _refused(bad, B.mmsp_cache_copy_pages, shape, cache, a["n_layers"], a["layer_stride"], a["copies"], a["n_copies"])
    _refused(B.MMSP_ERR_UNSUPPORTED, B.mmsp_cache_copy_pages, shape, _cache(page_size=1 << 24), 1, 0, FAKE, 1)


def test_calls_without_rows_do_nothing():
    """No GPU is here: a launch would come back as MMSP_ERR_DEVICE."""
    shape, cache = _shape(), _cache(n_seqs=0, n_rows=0, page_table=None, lengths=None)
    B.mmsp_cache_append(shape, cache, None, None, 0, FAKE, FAKE, FAKE, FAKE)
    B.mmsp_cache_attn(shape, cache, FAKE, FAKE, None, None, None, 0)
    B.mmsp_cache_copy_pages(shape, cache, 0, 0, FAKE, 3)
    B.mmsp_cache_copy_pages(shape, cache, 3, 8, None, 0)
    B.mmsp_rotary_apply(B.mmsp_rotary_plan(64, 1e4, [32]), 0, FAKE, 0, [B.make_heads(FAKE, 1, B.MMSP_F32, 64, 64)], [B.make_heads(FAKE, 1, B.MMSP_F32, 64, 64)])


# ---- page bookkeeping ----

class Server:
    """The bookkeeping beside a plain model: every page holds (sequence's) token numbers as text, copied as the calls say."""

    def __init__(self, n_pages, page_size, max_pages):
        self.refs, self.free_pages = np.zeros(n_pages, dtype=np.int32), np.zeros(n_pages, dtype=np.int32)
        self.pages = B.make_pages(self.refs, self.free_pages, page_size)
        self.max_pages, self.p = max_pages, page_size
        self.data = [[None] * page_size for _ in range(n_pages)]
        self.rows, self.text = {}, {}

    def copy(self, copies):
        src = [list(self.data[s]) for s, _, _ in copies]
        assert len({d for _, d, _ in copies}) == len(copies) and not {s for s, _, _ in copies} & {d for _, d, _ in copies}
        for (_, d, n), x in zip(copies, src):
            self.data[d][:n] = x[:n]

    def check(self):
        held = orc.Pages(len(self.refs), self.p)
        for s, row in self.rows.items():
            n = len(self.text[s])
            used = -(-n // self.p)
            held.held[s] = row[:used].tolist()
            assert [self.data[row[j // self.p]][j % self.p] for j in range(n)] == self.text[s]
            assert (row[used:] == -1).all() and len(set(held.held[s])) == used
        assert [held.holders(p) for p in range(len(self.refs))] == self.refs.tolist()
        assert sorted(self.free_pages[:self.pages.n_free].tolist()) == sorted(set(range(len(self.refs))) - held.used())


@pytest.mark.parametrize("seed", range(12))
def test_pages_against_a_plain_model(seed):
    rng = random.Random(seed)
    n_pages, p, max_pages = rng.choice([(7, 16, 5), (40, 16, 9), (64, 48, 30), (5, 1, 5)])
    m, names = Server(n_pages, p, max_pages), iter(range(10 ** 6))
    refused = compacted = copied = 0
    for step in range(300):
        what = rng.choice(["new", "grow", "grow", "grow", "fork", "free", "compact"])
        seqs = list(m.rows)
        if what == "new" or not seqs:
            s = next(names)
            m.rows[s], m.text[s] = np.full(max_pages, -1, dtype=np.int32), []
        elif what == "grow":
            s = rng.choice(seqs)
            old, more = len(m.text[s]), rng.choice([0, 1, 1, rng.randint(0, 3 * p)])
            state = m.refs.copy(), m.free_pages.copy(), m.pages.n_free, m.rows[s].copy()
            try:
                copy = B.mmsp_pages_grow(m.pages, m.rows[s], old, old + more)
            except B.MmspError as e:
                refused += e.status == B.MMSP_ERR_NO_PAGES
                assert e.status == (B.MMSP_ERR_NO_PAGES if -(-(old + more) // p) <= max_pages else B.MMSP_ERR_INVALID_ARG)
                now = m.refs, m.free_pages, m.pages.n_free, m.rows[s]
                assert all(np.array_equal(a, b) for a, b in zip(state, now))
                continue
            if copy is not None:
                copied += 1
                assert copy[2] == old % p
                m.copy([copy])
            for j in range(old, old + more):
                page = m.rows[s][j // p]
                assert m.refs[page] == 1                 # nobody else reads what is written
                m.data[page][j % p] = (s, j)
            m.text[s] = m.text[s] + [(s, j) for j in range(old, old + more)]
        elif what == "fork":
            s, t = rng.choice(seqs), next(names)
            m.rows[t] = np.zeros(max_pages, dtype=np.int32)
            B.mmsp_pages_fork(m.pages, m.rows[s], len(m.text[s]), m.rows[t])
            m.text[t] = list(m.text[s])
        elif what == "free":
            s = rng.choice(seqs)
            B.mmsp_pages_free(m.pages, m.rows[s], len(m.text[s]))
            assert (m.rows[s] == -1).all()
            del m.rows[s], m.text[s]
        else:
            table = np.stack([m.rows[s] for s in seqs])
            copies, used = B.mmsp_pages_compact(m.pages, table, np.array([len(m.text[s]) for s in seqs], dtype=np.int64))
            m.copy([tuple(c) for c in copies.tolist()])
            for s, row in zip(seqs, table):
                m.rows[s][:] = row
            compacted += len(copies)
            assert used == (m.refs > 0).sum() and (m.refs[:used] > 0).all()
        m.check()
    assert refused > 0 if n_pages < 40 else compacted > 0 and copied > 0     # a pool of a few pages is full or empty most of the time


def test_pages_refuse_and_change_nothing():
    refs, free = np.zeros(6, dtype=np.int32), np.zeros(6, dtype=np.int32)
    pages, row, bad = B.make_pages(refs, free, 16), np.full(4, -1, dtype=np.int32), B.MMSP_ERR_INVALID_ARG
    B.mmsp_pages_grow(pages, row, 0, 40)
    assert row.tolist() == [0, 1, 2, -1]
    other = np.full(4, -1, dtype=np.int32)
    B.mmsp_pages_fork(pages, row, 20, other)
    assert other.tolist() == [0, 1, -1, -1] and refs.tolist() == [2, 2, 1, 0, 0, 0]
    state = lambda: (refs.tolist(), free[:pages.n_free].tolist(), row.tolist(), other.tolist())
    before = state()
    wrong = np.array([0, 5, -1, -1], dtype=np.int32)     # page 5 is free
    twice = np.array([2, 2, -1, -1], dtype=np.int32)
    for f, *args in ((B.mmsp_pages_grow, row, 40, 30), (B.mmsp_pages_grow, row, 40, 65), (B.mmsp_pages_grow, row, -1, 4), (B.mmsp_pages_grow, wrong, 20, 21),
                     (B.mmsp_pages_free, wrong, 20), (B.mmsp_pages_free, twice, 20), (B.mmsp_pages_free, row, 65), (B.mmsp_pages_fork, wrong, 20, other),
                     (B.mmsp_pages_fork, row, 40, row)):
        _refused(bad, f, pages, *args)
        assert state() == before
    _refused(B.MMSP_ERR_NO_PAGES, B.mmsp_pages_grow, B.make_pages(np.zeros(1, dtype=np.int32), np.zeros(1, dtype=np.int32), 16), np.full(4, -1, dtype=np.int32), 0, 17)
    for table, lengths in ((np.stack([row]), [40]), (np.stack([row, other, other]), [40, 20, 20]), (np.stack([row, other]), [40, 16])):   # not all that is held, more, not all
        _refused(bad, B.mmsp_pages_compact, pages, table, np.array(lengths, dtype=np.int64))
        assert state() == before
    with pytest.raises(ValueError):
        B.mmsp_pages_grow(pages, row.astype(np.int64), 0, 1)
    with pytest.raises(ValueError):
        B.mmsp_pages_fork(pages, row, 20, other[:3].copy())


def test_pages_elsewhere_are_left_alone():
    """Entries of -1 among a sequence's pages: on another rank.  They are neither taken, shared, freed nor moved."""
    refs, free = np.zeros(8, dtype=np.int32), np.zeros(8, dtype=np.int32)
    pages, row, new = B.make_pages(refs, free, 16), np.full(6, -1, dtype=np.int32), np.zeros(6, dtype=np.int32)
    B.mmsp_pages_grow(pages, row, 0, 60)
    gone = np.array([row[0], -1], dtype=np.int32)        # its first page is let go of: the sequence keeps a hole
    B.mmsp_pages_free(pages, gone, 16)
    row[0] = -1
    B.mmsp_pages_fork(pages, row, 60, new)
    assert new.tolist() == row.tolist() == [-1, 1, 2, 3, -1, -1] and refs.tolist() == [0, 2, 2, 2, 0, 0, 0, 0]
    table = np.stack([row, new])
    copies, used = B.mmsp_pages_compact(pages, table, np.array([60, 60], dtype=np.int64))
    assert copies.tolist() == [[3, 0, 16]] and used == 3 and table.tolist() == [[-1, 1, 2, 0, -1, -1]] * 2
    row[:], new[:] = table
    assert B.mmsp_pages_grow(pages, new, 60, 61) == (0, pages_next(free, pages), 12)
    B.mmsp_pages_free(pages, row, 60)
    B.mmsp_pages_free(pages, new, 61)
    assert refs.tolist() == [0] * 8 and sorted(free.tolist()) == list(range(8)) and pages.n_free == 8


def pages_next(free, pages):
    """The page that was given out last."""
    return int(free[pages.n_free])


# ---- the layout of the attention ----

def _room(n_seqs, n_rows, most_new=0, cu_new=FAKE):
    """Bytes of partial results: they go by the rows of a group and the number of workgroups, the layout of the call."""
    shape = _shape(n_q_heads=28, n_kv_heads=4, q_strides=(3584, 128), kv_strides=(512, 128), lse_head_stride=n_rows)
    cache = _cache(page_size=64, max_pages=400, table_stride=400, n_seqs=n_seqs, n_rows=n_rows, cu_new=cu_new, most_new=most_new)
    return B.mmsp_cache_workspace_bytes(shape, cache) - -(-8 * n_rows * 28 // 16) * 16


def test_layouts_do_not_go_by_divisibility():
    """A total that the number of sequences happens to divide says nothing about the numbers of each."""
    assert _room(16, 31) == _room(16, 32) == _room(16, 33)
    assert _room(64, 191) == _room(64, 192) == _room(64, 193)
    assert _room(16, 79) == _room(16, 80) == _room(16, 81)


def test_layouts_go_by_the_most_new_tokens_of_a_sequence():
    one = _room(16, 16, cu_new=None)
    for pad in (0, 3, 16):                                  # padding rows change nothing where the number is known
        assert _room(16, 16 + pad, most_new=1) == one
        assert _room(16, 80 + pad, most_new=5) == _room(16, 80, most_new=5) == _room(1, 5) == _room(1, 5 + pad, most_new=5)
    assert _room(16, 32, most_new=2) == one != _room(16, 32)   # 14 rows a KV head, not 28
    assert _room(16, 80, most_new=500) == _room(16, 80)      # one long sequence among short ones: twice the mean at most
    assert _room(1, 40) == _room(1, 40, most_new=40)
    _refused(B.MMSP_ERR_INVALID_ARG, B.mmsp_cache_attn, _shape(), _cache(cu_new=FAKE, most_new=-1), FAKE, FAKE, None, None, FAKE, 1 << 40)


def test_a_step_says_how_many_new_tokens_its_sequences_have():
    import torch
    from paper_2408_10188_amd import paged
    c = paged.PagedCache(1, 12, 16, 4, 2, 128, 100, torch.bfloat16, "cpu")
    a, b = c.add(), c.add()
    c.step([a, b], [3, 5])
    assert c._cache(0).most_new == 5
    c.step([a], [1])
    assert c._cache(0).most_new == 1
