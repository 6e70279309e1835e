"""Inference over a paged key-value cache: descriptors for tensors, and `PagedCache`, the host side of a server's cache (all
layers' pools, the page tables of its sequences, and which pages are in use).  Like ring.py it only sequences C-ABI calls; the
arithmetic and the data movement happen in the kernels.

Pools are tensors [n_pages, n_kv_heads, page_size, d] of any strides with d contiguous (a transposed [n_pages, page_size,
n_kv_heads, d] is one).
"""
import numpy as np

from . import binding as B


def _io(t):
    import torch
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("bfloat16 or float32 is wanted, not %s" % t.dtype)
    return B.MMSP_F32 if t.dtype == torch.float32 else B.MMSP_BF16


def heads_of(t):
    """mmsp_heads of a tensor [rows, n_heads, d]."""
    if t.dim() != 3 or t.stride(2) != 1:
        raise ValueError("[rows, n_heads, d] with d contiguous is wanted")
    h = B.make_heads(t, t.shape[1], _io(t), *_strides(t))
    h.of = t.shape[0] if t.is_cuda else -1, t.shape[2]    # the calls check them
    return h


def shape_for(k_pool, io_dtype, n_q_heads=None, n_rows=0, scale=1.0):
    """mmsp_shape for a pool and dense rows of Q, K and V."""
    hkv, d = k_pool.shape[-3], k_pool.shape[-1]
    hq = hkv if n_q_heads is None else n_q_heads
    return B.make_shape(hq, hkv, d, io_dtype, scale, (hq * d, d), (hkv * d, d), n_rows)


def cache_for(k_pool, v_pool, page_table=None, lengths=None, n_rows=0, cu_new=None, most_new=0):
    """mmsp_cache for pools [n_pages, n_kv_heads, page_size, d], page_table [n_seqs, max_pages], lengths [n_seqs] and
    cu_new [n_seqs + 1] (int32, on the pool's device).  most_new: the most new tokens of a sequence, where cu_new is given and the host
    knows it; the attention is laid out by it (without it for up to twice the mean, which costs where all have the same number)."""
    import torch
    if (k_pool.dim() != 4 or k_pool.shape != v_pool.shape or k_pool.stride() != v_pool.stride() or k_pool.stride(3) != 1 or k_pool.dtype != v_pool.dtype
            or k_pool.device != v_pool.device):
        raise ValueError("two pools [n_pages, n_kv_heads, page_size, d] of the same type, strides and device, d contiguous, are wanted")
    for name, t, dims in (("page_table", page_table, 2), ("lengths", lengths, 1), ("cu_new", cu_new, 1)):
        if t is not None and (t.dtype != torch.int32 or t.dim() != dims or t.shape[-1] > 1 and t.numel() > 0 and t.stride(-1) != 1 or t.device != k_pool.device):
            raise ValueError("%s must be int32 with %d dimensions, contiguous, on the pool's device" % (name, dims))
    n_seqs = 0 if lengths is None else len(lengths)
    if page_table is not None and len(page_table) != n_seqs or cu_new is not None and len(cu_new) != n_seqs + 1:
        raise ValueError("page_table, lengths and cu_new must have n_seqs, n_seqs and n_seqs + 1 entries")
    if page_table is not None and n_seqs > 1 and page_table.stride(0) < page_table.shape[1]:
        raise ValueError("the rows of page_table must not overlap (an expanded one has to be copied)")
    pages, heads, page_size, d = k_pool.shape
    # a size of one may have any stride
    strides = (k_pool.stride(0) if pages > 1 else heads * page_size * d, k_pool.stride(2), k_pool.stride(1) if heads > 1 else page_size * d)
    width = 0 if page_table is None else page_table.shape[1]
    return B.make_cache(k_pool, v_pool, strides, pages, page_size, page_table, max(width, page_table.stride(0)) if width else 0, width, n_seqs, lengths,
                        cu_new, n_rows, most_new)


def _capturing(device):
    import torch
    return device.type == "cuda" and torch.cuda.is_current_stream_capturing()


class PagedCache:
    """The cache of a model's layers on one GPU: sequences are added, forked, extended and freed; pages are shared by forked
    sequences until one of them writes to its partly filled last page, and moved to the front of the pool on demand.

    Everything is enqueued on torch's current stream; calls on other streams are the caller's to order.  `step` says which new
    tokens come next; `append` and `attend` then run once per layer.

    None of it can be captured into a graph: a step's tables and workspace are new tensors that go with the next step, and a replay after that would read
    and write memory that others have by then.  A program that replays its steps keeps arrays of its own and makes the C calls."""

    def __init__(self, n_layers, n_pages, page_size, n_q_heads, n_kv_heads, head_dim, max_tokens, dtype, device="cuda"):
        import torch
        self.k, self.v = (torch.zeros(n_layers, n_pages, n_kv_heads, page_size, head_dim, dtype=dtype, device=device) for _ in range(2))
        self.page_size, self.n_q_heads, self.max_pages = page_size, n_q_heads, -(-max_tokens // page_size)
        self._refs, self._free = np.zeros(n_pages, dtype=np.int32), np.zeros(n_pages, dtype=np.int32)
        self.pages = B.make_pages(self._refs, self._free, page_size)
        self.rows, self.lengths, self._next = {}, {}, 0
        self._step = self._ws = None

    def _eager(self):
        if _capturing(self.k.device):
            raise RuntimeError("PagedCache cannot be captured into a graph: its arrays do not outlive a step (capture mmsp_cache_append and mmsp_cache_attn over arrays that stay)")

    def _add(self, row, length):
        self._next += 1
        self.rows[self._next], self.lengths[self._next] = row, length
        return self._next

    def add(self):
        """A new, empty sequence; returns its name."""
        return self._add(np.full(self.max_pages, -1, dtype=np.int32), 0)

    def fork(self, seq):
        """A second sequence with the same tokens so far, whose pages it shares."""
        row = np.full(self.max_pages, -1, dtype=np.int32)
        B.mmsp_pages_fork(self.pages, self.rows[seq], self.lengths[seq], row)
        return self._add(row, self.lengths[seq])

    def free(self, seq):
        B.mmsp_pages_free(self.pages, self.rows[seq], self.lengths[seq])
        del self.rows[seq], self.lengths[seq]
        if self._step is not None and seq in self._step[4]:
            self._step = None

    def _copy(self, copies):
        import torch
        if len(copies) == 0:
            return
        dev = torch.from_numpy(np.ascontiguousarray(copies, dtype=np.int32)).to(self.k.device)
        shape, cache = shape_for(self.k[0], _io(self.k)), cache_for(self.k[0], self.v[0])
        with torch.cuda.device(self.k.device):
            B.mmsp_cache_copy_pages(shape, cache, len(self.k), self.k.stride(0), dev, len(copies), torch.cuda.current_stream().cuda_stream)

    def compact(self):
        """Moves the pages in use to the front of the pool; returns how many there are.  Where the copies cannot be made it raises, and no page has moved."""
        self._eager()
        names = list(self.rows)
        table = np.stack([self.rows[s] for s in names]) if names else np.zeros((0, self.max_pages), dtype=np.int32)
        before = self._refs.copy(), self._free.copy(), self.pages.n_free
        copies, used = B.mmsp_pages_compact(self.pages, table, np.array([self.lengths[s] for s in names], dtype=np.int64))
        try:
            self._copy(copies)
        except BaseException:                             # copies that were made went into free pages
            self._refs[:], self._free[:], self.pages.n_free = before
            raise
        for s, row in zip(names, table):
            self.rows[s][:] = row
        self._step = None
        return used

    def step(self, seqs, n_new):
        """The next n_new[i] tokens of sequences seqs[i], whose rows of Q, K and V come one sequence after the other.  Takes the
        pages for them; raises MmspError (status MMSP_ERR_NO_PAGES) where the pool has too few.  A call that raises, for whatever
        reason, has changed nothing: the step before it is still the present one."""
        import torch
        self._eager()
        if len(set(seqs)) != len(seqs) or len(seqs) != len(n_new) or min(n_new, default=0) < 0:
            raise ValueError("every sequence once, with a number of new tokens")
        copies, done = [], []
        try:
            for s, n in zip(seqs, n_new):
                before = self.rows[s].copy()
                copy = B.mmsp_pages_grow(self.pages, self.rows[s], self.lengths[s], self.lengths[s] + n)
                done.append((s, n, before))
                if copy is not None:
                    copies.append(copy)
            dev = self.k.device
            after = [self.lengths[s] + n for s, n in zip(seqs, n_new)]
            # as wide as the longest of them: the calls lay their work out for that many tokens
            width = max([1] + [-(-n // self.page_size) for n in after])
            table = torch.from_numpy(np.stack([self.rows[s][:width] for s in seqs]) if seqs else np.zeros((0, width), dtype=np.int32)).to(dev)
            lengths = torch.tensor(after, dtype=torch.int32, device=dev)
            cu_new = None if all(n == 1 for n in n_new) else torch.from_numpy(np.concatenate([[0], np.cumsum(n_new)]).astype(np.int32)).to(dev)
            self._copy(copies)
        except BaseException:
            for s, n, before in reversed(done):           # what was taken is given back; copies into it, if some were made, change nothing that is held
                self._undo(s, n, before)
            raise
        self.lengths.update(zip(seqs, after))
        self._step = (table, lengths, cu_new, int(sum(n_new)), frozenset(seqs), int(max(n_new, default=0)))
        self._ws = None

    def _undo(self, seq, n, before):
        now, old = self.rows[seq], self.lengths[seq]
        have, first = -(-old // self.page_size), -(-old // self.page_size)
        if have and before[have - 1] != now[have - 1]:    # the page of its own goes, the shared one comes back
            self._refs[before[have - 1]] += 1
            first -= 1
        taken = now[first:-(-(old + n) // self.page_size)].copy()
        B.mmsp_pages_free(self.pages, taken, len(taken) * self.page_size)
        now[:] = before

    def _cache(self, layer):
        if self._step is None:
            raise RuntimeError("step() comes first")
        table, lengths, cu_new, n_rows, _, most_new = self._step
        return cache_for(self.k[layer], self.v[layer], table, lengths, n_rows, cu_new, most_new)

    def _shape(self, q, k=None, scale=1.0):
        d = self.k.shape[-1]
        hkv = self.k.shape[2]
        strides = (hkv * d, d) if k is None else _strides(k)
        return B.make_shape(self.n_q_heads, hkv, d, _io(self.k), scale, _strides(q), strides, q.shape[0])

    def append(self, layer, rotary, positions, q, k, v, q_out=None):
        """Writes the step's K (turned by `rotary` at `positions` [n_axes, rows]) and V into `layer`'s pages; returns Q turned (into q_out:
        contiguous, or q itself, which is also what None means)."""
        import torch
        self._eager()
        cache, n = self._cache(layer), self._step[3]
        q_out = q if q_out is None else q_out
        for t in (q, k, v, q_out):
            if t.dim() != 3 or t.shape[0] != n or t.dtype != self.k.dtype or t.stride(2) != 1 or t.device != self.k.device:
                raise ValueError("%d rows of %s with d contiguous, on the pool's device, are wanted" % (n, self.k.dtype))
        if _strides(k) != _strides(v) or k.shape != v.shape or q.shape != q_out.shape:
            raise ValueError("K and V must have the same shapes and strides, q_out Q's shape")
        if q_out.stride() != q.stride() if q_out.data_ptr() == q.data_ptr() else not q_out.is_contiguous():
            raise ValueError("q_out must be contiguous, or q itself")
        if q.shape[1:] != (self.n_q_heads, self.k.shape[-1]) or k.shape[1:] != (self.k.shape[2], self.k.shape[-1]):
            raise ValueError("Q and K must have the cache's heads")
        if rotary is not None and (positions is None or positions.dtype != torch.int32 or positions.shape != (rotary.n_axes, n) or n > 1 and positions.stride(1) != 1
                                   or rotary.n_axes > 1 and positions.stride(0) < n or positions.device != self.k.device):
            raise ValueError("positions must be int32 [%d, %d] on the pool's device, contiguous, the axes apart (expanded ones have to be copied)" % (rotary.n_axes, n))
        if n == 0:
            return q_out
        with torch.cuda.device(self.k.device):
            B.mmsp_cache_append(self._shape(q, k), cache, rotary, positions, 0 if positions is None else max(n, positions.stride(0)), q, k, v, q_out,
                                torch.cuda.current_stream().cuda_stream)
        return q_out

    def attend(self, layer, q, scale=None, o_final=None, o=None, lse=None):
        """Attention of the step's rows over `layer`'s cache: O in q's type (into o_final, made if nothing is given), or the
        partial result (o, lse) for mmsp_attn_merge.  Dense [rows, n_q_heads, d] and [n_q_heads, rows]."""
        import torch
        self._eager()
        cache, n = self._cache(layer), self._step[3]
        if q.shape != (n, self.n_q_heads, self.k.shape[-1]) or q.dtype != self.k.dtype or q.stride(2) != 1 or q.device != self.k.device:
            raise ValueError("q must be %s [%d, %d, %d] on the pool's device" % (self.k.dtype, n, self.n_q_heads, self.k.shape[-1]))
        if o_final is None and o is None:
            o_final = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        for t, dtype, size in ((o_final, q.dtype, tuple(q.shape)), (o, torch.float32, tuple(q.shape)), (lse, torch.float32, (self.n_q_heads, n))):
            if t is not None and (t.dtype != dtype or tuple(t.shape) != size or not t.is_contiguous() or t.device != q.device):
                raise ValueError("results must be contiguous, on q's device, o_final in q's type, o and lse in float32")
        if n == 0:
            return o_final if o_final is not None else (o, lse)
        shape = self._shape(q, scale=q.shape[-1] ** -0.5 if scale is None else scale)
        if self._ws is None:                              # one for all layers of a step: they run one after the other
            self._ws = torch.empty(max(B.mmsp_cache_workspace_bytes(shape, cache), 16), dtype=torch.uint8, device=q.device)
        with torch.cuda.device(q.device):
            B.mmsp_cache_attn(shape, cache, q, o_final, o, lse, self._ws, self._ws.numel(), torch.cuda.current_stream().cuda_stream)
        return o_final if o_final is not None else (o, lse)


def _strides(t):
    """Token and head stride; a size of one may have any."""
    d = t.shape[2]
    return (t.stride(0) if t.shape[0] > 1 else max(t.stride(0), d) // 8 * 8, t.stride(1) if t.shape[1] > 1 else d)
