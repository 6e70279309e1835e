"""The host side of the cache's Python layer, and that its structures are the header's.  No kernel is launched here."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2408_10188_amd import binding as B
from paper_2408_10188_amd import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_structures_are_laid_out_as_in_the_header(tmp_path):
    structs = dict(mmsp_rotary=B.MmspRotary, mmsp_heads=B.MmspHeads, mmsp_cache=B.MmspCache, mmsp_page_copy=B.MmspPageCopy, mmsp_pages=B.MmspPages)
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "mmsp.h"', "int main(void) {"]
    for name, s in structs.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in s._fields_]
    (tmp_path / "a.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(tmp_path / "a.c"), "-o", str(tmp_path / "a")], check=True)
    said = dict(ln.split() for ln in subprocess.run([str(tmp_path / "a")], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, s in structs.items():
        assert int(said[name]) == ctypes.sizeof(s)
        for f, _ in s._fields_:
            assert int(said["%s.%s" % (name, f)]) == getattr(s, f).offset, (name, f)


@pytest.mark.parametrize("first", ["from paper_2408_10188_amd import binding", "import torch"])
def test_one_hip_runtime_in_whatever_order(first):
    """The library and torch share one, also where the binding is imported before torch."""
    code = first + "\nimport torch\nfrom paper_2408_10188_amd import binding\nprint(len({line.split()[-1] for line in open('/proc/self/maps') if 'libamdhip64' in line}))"
    assert subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True, capture_output=True, text=True).stdout.split() == ["1"]


def _cache(n_pages=12, page=16, max_tokens=100):
    return paged.PagedCache(2, n_pages, page, 4, 2, 128, max_tokens, torch.bfloat16, "cpu")


def _state(c):
    return c._refs.tolist(), c.pages.n_free, {s: r.tolist() for s, r in c.rows.items()}, dict(c.lengths)


def test_steps_take_pages_all_or_none():
    c = _cache()
    a, b = c.add(), c.add()
    c.step([a, b], [40, 16])
    assert c.rows[a].tolist() == [0, 1, 2, -1, -1, -1, -1] and c.rows[b][:2].tolist() == [3, -1] and c.lengths == {a: 40, b: 16}
    table, lengths, cu_new, n = c._step[:4]
    assert table.tolist() == [c.rows[a][:3].tolist(), c.rows[b][:3].tolist()] and lengths.tolist() == [40, 16] and cu_new.tolist() == [0, 40, 56] and n == 56
    c.step([b], [1])
    assert c._step[2] is None and c.rows[b][:2].tolist() == [3, 4]
    fork = c.fork(a)                                     # its last page is half full and shared
    before = _state(c)
    for seqs, n_new, error in (([b, fork, a], [64, 20, 60], B.MmspError), ([b, a], [70, 100], B.MmspError), ([fork, 99], [30, 1], KeyError),
                               ([a, a], [1, 1], ValueError), ([a], [1, 2], ValueError), ([a], [-1], ValueError)):
        with pytest.raises(error):
            c.step(seqs, n_new)
        assert _state(c) == before
        assert sorted(c._free[:c.pages.n_free].tolist()) == [i for i, r in enumerate(before[0]) if r == 0]
    c.free(a)
    c.step([fork], [8])                                  # nobody else holds its last page any more: no copy is made
    assert c.rows[fork][:3].tolist() == [0, 1, 2]
    c.free(fork)
    assert c.pages.n_free == 10 and sorted(np.flatnonzero(c._refs)) == [3, 4] and list(c.rows) == [b]
    c.free(b)
    assert c.pages.n_free == 12 and c.compact() == 0


def test_compaction_of_an_empty_cache():
    c = _cache()
    assert c.compact() == 0
    with pytest.raises(RuntimeError):
        c.attend(0, torch.zeros(1, 4, 128, dtype=torch.bfloat16))


def test_layers_of_the_python_side_refuse_wrong_tensors():
    c = _cache()
    a = c.add()
    c.step([a], [3])
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    rot = B.mmsp_rotary_plan(128, 1e6, [16, 24, 24])
    pos = torch.zeros(3, 3, dtype=torch.int32)
    good = dict(q=bf(3, 4, 128), k=bf(3, 2, 128), v=bf(3, 2, 128), q_out=None)
    wide = bf(3, 8, 128)
    for kw in (dict(q=bf(2, 4, 128)), dict(q=bf(3, 5, 128)), dict(k=bf(3, 3, 128), v=bf(3, 3, 128)), dict(v=wide[:, :2]), dict(q=torch.zeros(3, 4, 128)), dict(q=wide[:, :4].to("meta")),
               dict(q_out=wide[:, :4]), dict(q=wide[:, :4], q_out=wide.view(-1)[:3 * 512].view(3, 4, 128))):
        with pytest.raises(ValueError):
            c.append(0, rot, pos, **{**good, **kw})
    for p in (None, pos[:2], pos.long(), torch.zeros(3, 4, dtype=torch.int32), pos.to("meta"), pos[:1].expand(3, 3), pos.T):
        with pytest.raises(ValueError):
            c.append(0, rot, p, **good)
    for kw in (dict(q=bf(3, 2, 128)), dict(o_final=torch.zeros(3, 4, 128)), dict(o=bf(3, 4, 128)), dict(o_final=wide[:, :4]), dict(lse=torch.zeros(4, 4)), dict(q=bf(3, 4, 128).to("meta"))):
        with pytest.raises(ValueError):
            c.attend(0, **{**dict(q=bf(3, 4, 128)), **kw})
    pool = torch.zeros(4, 2, 16, 128)
    for bad in (dict(v_pool=pool.bfloat16()), dict(v_pool=pool[:3]), dict(v_pool=pool.to("meta")),
                dict(page_table=torch.zeros(1, 2, dtype=torch.int32).expand(3, 2), lengths=torch.zeros(3, dtype=torch.int32)), dict(page_table=torch.zeros(1, 2)), dict(lengths=torch.zeros(1)),
                dict(page_table=torch.zeros(2, 2, dtype=torch.int32), lengths=torch.zeros(1, dtype=torch.int32)),
                dict(lengths=torch.zeros(2, dtype=torch.int32), cu_new=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            paged.cache_for(**{**dict(k_pool=pool, v_pool=pool), **bad})
    assert paged.heads_of(torch.zeros(3, 260, dtype=torch.bfloat16)[:1, :256].view(1, 2, 128)).tok_stride % 8 == 0
    with pytest.raises(ValueError):
        paged.heads_of(torch.zeros(3, 128, 4).transpose(1, 2))
    with pytest.raises(ValueError):
        paged.heads_of(torch.zeros(3, 4, 128, dtype=torch.float16))


def test_a_sequence_that_goes_ends_the_step_it_is_in():
    c = _cache()
    a, b = c.add(), c.add()
    c.step([b], [3])
    c.free(a)
    assert c._cache(0).n_rows == 3
    c.free(b)
    with pytest.raises(RuntimeError):
        c._cache(0)


def test_a_step_without_tokens_does_nothing():
    c = _cache()
    a = c.add()
    c.step([a], [0])
    empty = torch.zeros(0, 4, 128, dtype=torch.bfloat16)
    kv = torch.zeros(0, 2, 128, dtype=torch.bfloat16)
    assert c.append(0, None, None, empty, kv, kv) is empty and c.attend(0, empty).shape == (0, 4, 128)
    c.step([], [])


def test_calls_too_large_for_a_grid_are_refused():
    shape = B.make_shape(4, 2, 128, B.MMSP_BF16, 0.1, (512, 128), (256, 128), 1024)
    cache = lambda n, pages: B.make_cache(4096, 4096, (4096, 128, 2048), 9, 16, 4096, pages, pages, n, 4096, None, n)
    assert B.mmsp_cache_workspace_bytes(shape, cache(60, 1 << 26)) > 0
    for n, pages in ((64, 1 << 26), (1 << 20, 1 << 17)):                    # 2^30 tokens each; 2^21, and a million sequences
        with pytest.raises(B.MmspError) as e:
            B.mmsp_cache_attn(B.make_shape(4, 2, 128, B.MMSP_BF16, 0.1, (512, 128), (256, 128), 1 << 20), cache(n, pages), 4096, 4096, None, None, 4096, 1 << 50)
        assert e.value.status == B.MMSP_ERR_UNSUPPORTED
    with pytest.raises(B.MmspError) as e:                                   # 2^22 layers of K and V of 512 pieces of 16 bytes: 2^32 threads
        B.mmsp_cache_copy_pages(shape, cache(1, 1), 1 << 22, 8, 4096, 1)
    assert e.value.status == B.MMSP_ERR_UNSUPPORTED


def _fails(*args, **kw):
    raise MemoryError("no room on the device")


@pytest.mark.parametrize("what", ["the copies", "the table", "the lengths"])
def test_a_step_whose_device_work_fails_changes_nothing(what, monkeypatch):
    """Where the uploads or the page copies raise, no page has been taken and no length moved; the next step makes the copy that this one did not."""
    c = _cache()
    a = c.add()
    c.step([a], [20])
    b = c.fork(a)                                        # its second page is partly filled and shared
    before, step = _state(c), c._step
    with monkeypatch.context() as m:
        if what == "the copies":
            m.setattr(c, "_copy", _fails)
        else:
            m.setattr(torch, "from_numpy" if what == "the table" else "tensor", _fails)
        with pytest.raises(MemoryError):
            c.step([b, a], [30, 1])
    assert _state(c) == before and c._step is step
    assert sorted(c._free[:c.pages.n_free].tolist()) == [i for i, r in enumerate(before[0]) if r == 0]
    made = []
    monkeypatch.setattr(c, "_copy", made.extend)
    c.step([b], [1])
    assert made == [(1, c.rows[b][1], 4)] and c.rows[b][1] not in before[2][a] and c.lengths == {a: 20, b: 21}


def test_a_compaction_whose_copies_fail_moves_nothing(monkeypatch):
    c = _cache()
    a, b = c.add(), c.add()
    c.step([a, b], [40, 20])
    c.free(a)
    c.step([b], [1])
    before, free, step = _state(c), c._free.tolist(), c._step
    with monkeypatch.context() as m:
        m.setattr(c, "_copy", _fails)
        with pytest.raises(MemoryError):
            c.compact()
    assert _state(c) == before and c._free.tolist() == free and c._step is step
    made = []
    monkeypatch.setattr(c, "_copy", lambda copies: made.extend(copies.tolist()))
    assert c.compact() == 2 and made == [[3, 0, 16], [4, 1, 16]] and c.rows[b][:2].tolist() == [0, 1]
    with pytest.raises(RuntimeError):
        c._cache(0)


def test_a_step_of_no_sequences_is_one_without_rows():
    c = _cache()
    c.step([], [])
    q, kv = torch.zeros(0, 4, 128, dtype=torch.bfloat16), torch.zeros(0, 2, 128, dtype=torch.bfloat16)
    assert c.append(0, None, None, q, kv, kv) is q and c.attend(0, q).shape == (0, 4, 128)
    # a size of one, or of none, may have any stride
    pool = torch.zeros(4, 2, 16, 128)
    ints = torch.zeros(6, dtype=torch.int32)
    assert paged.cache_for(pool, pool.clone(), ints[::3].view(2, 1)[:1], ints[::2][:1]).n_seqs == 1
    assert paged.cache_for(pool, pool.clone(), ints[::3].view(2, 1), ints[:2]).table_stride == 3


class _OnGpu:
    """What the binding asks of a tensor of positions, as if it lay on a GPU."""

    def __init__(self, t):
        self.t, self.is_cuda = t, True

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_rotary_calls_refuse_tensors_that_are_not_what_the_kernel_reads():
    """Positions of another type or elsewhere, or too few; Q and K elsewhere, of fewer rows or a smaller head.  (All would be read as they lie.)"""
    rot = B.mmsp_rotary_plan(128, 1e6, [16, 24, 24])
    fake = lambda: B.make_heads(4096, 4, B.MMSP_BF16, 512, 128)
    pos = torch.zeros(3, 5, dtype=torch.int32)
    shape = B.make_shape(4, 2, 128, B.MMSP_BF16, 0.1, (512, 128), (256, 128), 5)
    cache = B.make_cache(4096, 4096, (4096, 128, 2048), 9, 16, 4096, 4, 4, 5, 4096, None, 5)
    for p, stride in ((pos, 5), (_OnGpu(pos.long()), 5), (_OnGpu(pos.float()), 5), (_OnGpu(pos[:2].clone()), 5), (_OnGpu(pos), 6), (_OnGpu(pos[:, 1:]), 5)):
        with pytest.raises(ValueError):
            B.mmsp_rotary_apply(rot, 5, p, stride, [fake()], [fake()])
        with pytest.raises(ValueError):
            B.mmsp_cache_append(shape, cache, rot, p, stride, 4096, 4096, 4096, 4096)
    B._positions(rot, 4, _OnGpu(pos[:, 1:]), 5)              # columns of a wider tensor reach to its end
    B._positions(rot, 5, _OnGpu(pos), 5)
    on_cpu = paged.heads_of(torch.zeros(5, 4, 128, dtype=torch.bfloat16))
    few, narrow = fake(), fake()
    few.of, narrow.of = (4, 128, True), (5, 64, True)
    for h in (on_cpu, few, narrow):
        for x, y in ((h, fake()), (fake(), h)):
            with pytest.raises(ValueError):
                B.mmsp_rotary_apply(rot, 5, _OnGpu(pos), 5, [fake(), x], [fake(), y])


def test_calls_under_capture_are_refused(monkeypatch):
    """A graph would go on reading a step's arrays after the next step has let go of them."""
    c = _cache()
    a, b = c.add(), c.add()
    c.step([a, b], [3, 20])
    c.free(a)
    before, step = _state(c), c._step
    q, kv = torch.zeros(3, 4, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    with monkeypatch.context() as m:
        m.setattr(paged, "_capturing", lambda device: True)
        for call in (lambda: c.step([b], [1]), c.compact, lambda: c.append(0, None, None, q, kv, kv), lambda: c.attend(0, q)):
            with pytest.raises(RuntimeError, match="captured"):
                call()
    assert _state(c) == before and c._step is step
    c.step([b], [1])


def test_the_binding_alone_does_not_import_torch():
    """A host program that plans layouts or pages does not pay for torch's start."""
    code = "from paper_2408_10188_amd import binding, paged\nimport sys\nprint('torch' in sys.modules, binding.mmsp_zigzag_layout(64, 4, 0, False)[0])"
    assert subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True, capture_output=True, text=True).stdout.split() == ["False", "(0,", "7)"]


def test_page_copies_refuse_lists_that_are_not_what_the_kernel_reads():
    shape, cache = B.make_shape(4, 2, 128, B.MMSP_BF16, 0.1, (512, 128), (256, 128), 5), B.make_cache(4096, 4096, (4096, 128, 2048), 9, 16)
    copies = torch.zeros(4, 3, dtype=torch.int32)
    for x, n in ((copies, 4), (_OnGpu(copies.long()), 4), (_OnGpu(copies), 5), (_OnGpu(copies.t()), 4), (_OnGpu(copies[:, :2]), 2)):
        with pytest.raises(ValueError):
            B.mmsp_cache_copy_pages(shape, cache, 1, 0, x, n)
    B.mmsp_cache_copy_pages(shape, cache, 1, 0, _OnGpu(copies), 0)
