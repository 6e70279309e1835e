"""ctypes binding of libmmsp.so: the same calls as include/mmsp.h, argument marshalling only.

Tensors are anything with `.data_ptr()` (torch tensors on the GPU); PyTorch is used by the
callers for device memory and streams, never for arithmetic on the attention path.
There is no fallback: if the library has not been built, importing this module raises.
"""
import ctypes
import importlib.util
import os
import sys

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmmsp.so")

MMSP_OK, MMSP_ERR_INVALID_ARG, MMSP_ERR_UNSUPPORTED, MMSP_ERR_WORKSPACE_TOO_SMALL, MMSP_ERR_DEVICE, MMSP_ERR_NO_PAGES = range(6)
MMSP_MASK_FULL, MMSP_MASK_CAUSAL_DIAG, MMSP_MASK_NONE = 0, 1, 2
MMSP_BF16, MMSP_F32 = 0, 1

EXPORTS = ["mmsp_zigzag_layout", "mmsp_zigzag_plan", "mmsp_contiguous_plan", "mmsp_zigzag_plan_packed", "mmsp_2d_layout", "mmsp_workspace_bytes", "mmsp_attn_step_fwd",
           "mmsp_attn_merge", "mmsp_attn_delta", "mmsp_attn_step_bwd", "mmsp_attn_step_bwd_static", "mmsp_zigzag_gather", "mmsp_zigzag_scatter",
           "mmsp_a2a_pack_heads", "mmsp_a2a_unpack_heads", "mmsp_rotary_plan", "mmsp_rotary_apply", "mmsp_cache_append", "mmsp_cache_workspace_bytes",
           "mmsp_cache_attn", "mmsp_cache_copy_pages", "mmsp_pages_init", "mmsp_pages_grow", "mmsp_pages_fork", "mmsp_pages_free", "mmsp_pages_compact",
           "mmsp_last_error"]


class MmspShape(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("io_dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("q_tok_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("kv_tok_stride", ctypes.c_int64), ("kv_head_stride", ctypes.c_int64),
                ("lse_head_stride", ctypes.c_int64)]


class MmspBlock(ctypes.Structure):
    _fields_ = [("q_row0", ctypes.c_int64), ("n_q", ctypes.c_int64), ("k_row0", ctypes.c_int64),
                ("n_k", ctypes.c_int64), ("q_pos0", ctypes.c_int64), ("k_pos0", ctypes.c_int64),
                ("mask", ctypes.c_int32), ("n_docs", ctypes.c_int32), ("cu_seqlens", ctypes.c_void_p)]


class Mmsp2dShare(ctypes.Structure):
    _fields_ = [("head_rank", ctypes.c_int32), ("ring_rank", ctypes.c_int32), ("q_head0", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("kv_head0", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("chunk_ids", ctypes.c_int32 * 2), ("chunk_len", ctypes.c_int64)]


class MmspRotary(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("turns", ctypes.c_uint64 * 64), ("axis", ctypes.c_uint8 * 64)]


class MmspHeads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n_heads", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("tok_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]
    of = None                                             # of a tensor: the rows that a call may have (-1: it is not on a GPU), and its head_dim


class MmspCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("tok_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("page_table", ctypes.c_void_p),
                ("table_stride", ctypes.c_int64), ("max_pages", ctypes.c_int32), ("n_seqs", ctypes.c_int32), ("lengths", ctypes.c_void_p),
                ("cu_new", ctypes.c_void_p), ("n_rows", ctypes.c_int32), ("most_new", ctypes.c_int32)]


class MmspPageCopy(ctypes.Structure):
    _fields_ = [("src", ctypes.c_int32), ("dst", ctypes.c_int32), ("n_tokens", ctypes.c_int32)]


class MmspPages(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("refs", ctypes.POINTER(ctypes.c_int32)),
                ("free_pages", ctypes.POINTER(ctypes.c_int32)), ("n_free", ctypes.c_int32)]


class MmspError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("mmsp status %d: %s" % (status, message))
        self.status = status


if not os.path.exists(LIB_PATH):
    raise ImportError("libmmsp.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                      "(or python paper_2408_10188_amd/build.py) first; there is no fallback path")


def _one_hip_runtime():
    """torch brings a HIP runtime of its own, which the library shares if it is there first; loaded the other way round there are two in the
    process, and the one behind the library sees no device.  The runtime alone is loaded here: a program that only plans layouts or pages does not wait for torch."""
    spec = importlib.util.find_spec("torch")
    path = os.path.join(os.path.dirname(spec.origin), "lib", "libamdhip64.so") if spec is not None and spec.origin else ""
    if os.path.exists(path):
        ctypes.CDLL(path)


_one_hip_runtime()
_lib = ctypes.CDLL(LIB_PATH)

_P, _I64, _I32, _INT, _SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int, ctypes.c_size_t
_lib.mmsp_last_error.restype = ctypes.c_char_p
_lib.mmsp_last_error.argtypes = []
_lib.mmsp_zigzag_layout.argtypes = [_I64, _I32, _I32, ctypes.POINTER(_I32), ctypes.POINTER(_I64)]
_lib.mmsp_zigzag_plan.argtypes = [_I64, _I32, _I32, _I32, ctypes.POINTER(_I32), ctypes.POINTER(MmspBlock)]
_lib.mmsp_contiguous_plan.argtypes = [_I64, _I32, _I32, _I32, ctypes.POINTER(_I32), ctypes.POINTER(MmspBlock)]
_lib.mmsp_zigzag_plan_packed.argtypes = [_I64, _I32, _I32, _I32, ctypes.POINTER(_I32), _I32, ctypes.POINTER(_I32),
                                         ctypes.POINTER(MmspBlock), ctypes.POINTER(_I32)]
_lib.mmsp_2d_layout.argtypes = [_I64, _I32, _I32, _I32, _I32, _I32, ctypes.POINTER(Mmsp2dShare)]
_lib.mmsp_zigzag_gather.argtypes = [_I64, _I32, _I64, _P, _P, _P]
_lib.mmsp_zigzag_scatter.argtypes = [_I64, _I32, _I64, _P, _P, _P]
_lib.mmsp_a2a_pack_heads.argtypes = [_I64, _I32, _I64, _P, _P, _P]
_lib.mmsp_a2a_unpack_heads.argtypes = [_I64, _I32, _I64, _P, _P, _P]
_lib.mmsp_workspace_bytes.restype = _SZ
_lib.mmsp_workspace_bytes.argtypes = [ctypes.POINTER(MmspShape), _I64, _I64, _INT]
_lib.mmsp_attn_step_fwd.argtypes = [ctypes.POINTER(MmspShape), ctypes.POINTER(MmspBlock), _P, _P, _P, _P, _P, _INT,
                                    _P, _SZ, _P]
_lib.mmsp_attn_merge.argtypes = [ctypes.POINTER(MmspShape), _I64, _I64, _P, _P, _P, _P, _P, _P]
_lib.mmsp_attn_delta.argtypes = [ctypes.POINTER(MmspShape), _I64, _I64, _P, _P, _P, _P]
_lib.mmsp_attn_step_bwd.argtypes = [ctypes.POINTER(MmspShape), ctypes.POINTER(MmspBlock), _P, _P, _P, _P, _P, _P, _P,
                                    _INT, _P, _P, _P, _INT, _P, _SZ, _P]
_lib.mmsp_attn_step_bwd_static.argtypes = [ctypes.POINTER(MmspShape), ctypes.POINTER(MmspBlock), _P, _P, _P, _P, _P, _P,
                                           _P, _INT, _P, _P, _P, _INT, _P]
_ROT, _HEADS, _CACHE, _PAGES, _IP = (ctypes.POINTER(x) for x in (MmspRotary, MmspHeads, MmspCache, MmspPages, _I32))
_COPY = ctypes.POINTER(MmspPageCopy)
_lib.mmsp_rotary_plan.argtypes = [_I32, ctypes.c_double, _I32, _IP, _ROT]
_lib.mmsp_rotary_apply.argtypes = [_ROT, _I64, _P, _I64, _I32, _HEADS, _HEADS, _INT, _P]
_lib.mmsp_cache_append.argtypes = [ctypes.POINTER(MmspShape), _CACHE, _ROT, _P, _I64, _P, _P, _P, _P, _P]
_lib.mmsp_cache_workspace_bytes.restype = _SZ
_lib.mmsp_cache_workspace_bytes.argtypes = [ctypes.POINTER(MmspShape), _CACHE]
_lib.mmsp_cache_attn.argtypes = [ctypes.POINTER(MmspShape), _CACHE, _P, _P, _P, _P, _P, _SZ, _P]
_lib.mmsp_cache_copy_pages.argtypes = [ctypes.POINTER(MmspShape), _CACHE, _I32, _I64, _P, _I32, _P]
_lib.mmsp_pages_init.argtypes = [_PAGES]
_lib.mmsp_pages_grow.argtypes = [_PAGES, _IP, _I32, _I64, _I64, _COPY, _IP]
_lib.mmsp_pages_fork.argtypes = [_PAGES, _IP, _I32, _I64, _IP]
_lib.mmsp_pages_free.argtypes = [_PAGES, _IP, _I32, _I64]
_lib.mmsp_pages_compact.argtypes = [_PAGES, _IP, _I64, _I32, _I32, ctypes.POINTER(_I64), _COPY, _IP, _IP]
for _name in EXPORTS:
    if _name not in ("mmsp_last_error", "mmsp_workspace_bytes", "mmsp_cache_workspace_bytes"):
        getattr(_lib, _name).restype = _INT


def _ptr(t):
    return None if t is None else (t if isinstance(t, int) else t.data_ptr())


def _check(status):
    if status != MMSP_OK:
        raise MmspError(status, _lib.mmsp_last_error().decode())


def mmsp_last_error():
    return _lib.mmsp_last_error().decode()


def make_shape(n_q_heads, n_kv_heads, head_dim, io_dtype, softmax_scale, q_strides, kv_strides, lse_head_stride):
    """q_strides / kv_strides = (token stride, head stride) in elements."""
    return MmspShape(n_q_heads, n_kv_heads, head_dim, io_dtype, softmax_scale, q_strides[0], q_strides[1],
                     kv_strides[0], kv_strides[1], lse_head_stride)


def make_block(q_row0, n_q, k_row0, n_k, mask, q_pos0=0, k_pos0=0, cu_seqlens=None, n_docs=0):
    return MmspBlock(q_row0, n_q, k_row0, n_k, q_pos0, k_pos0, mask, n_docs, _ptr(cu_seqlens))


def mmsp_zigzag_layout(T, N, rank, want_map=True):
    ids = (_I32 * 2)()
    l2g = np.empty(T // N if (N > 0 and T > 0) else 0, dtype=np.int64) if want_map else None
    p = l2g.ctypes.data_as(ctypes.POINTER(_I64)) if want_map else None
    _check(_lib.mmsp_zigzag_layout(T, N, rank, ids, p))
    return (ids[0], ids[1]), l2g


def mmsp_zigzag_plan(T, N, rank, step):
    src = _I32()
    blk = MmspBlock()
    _check(_lib.mmsp_zigzag_plan(T, N, rank, step, ctypes.byref(src), ctypes.byref(blk)))
    return src.value, blk


def mmsp_contiguous_plan(T, N, rank, step):
    src = _I32()
    blk = MmspBlock()
    _check(_lib.mmsp_contiguous_plan(T, N, rank, step, ctypes.byref(src), ctypes.byref(blk)))
    return src.value, blk


def mmsp_zigzag_plan_packed(T, N, rank, step, cu_seqlens=None, n_docs=0, cu_host=None):
    """Returns (src, [blocks]); cu_seqlens (device int32 tensor) / n_docs are filled into every
    block; cu_host (numpy int32 copy of cu_seqlens) lets the plan drop segment pairs no document spans."""
    src, n = _I32(), _I32()
    blks = (MmspBlock * 4)()
    hp, hn = None, 0
    if cu_host is not None:
        cu_host = np.ascontiguousarray(cu_host, dtype=np.int32)
        hp, hn = cu_host.ctypes.data_as(ctypes.POINTER(_I32)), len(cu_host) - 1
    _check(_lib.mmsp_zigzag_plan_packed(T, N, rank, step, hp, hn, ctypes.byref(src), blks, ctypes.byref(n)))
    out = []
    for i in range(n.value):
        b = MmspBlock.from_buffer_copy(blks[i])
        b.cu_seqlens, b.n_docs = _ptr(cu_seqlens), n_docs
        out.append(b)
    return src.value, out


def mmsp_2d_layout(T, U, R, gpu, n_q_heads, n_kv_heads):
    share = Mmsp2dShare()
    _check(_lib.mmsp_2d_layout(T, U, R, gpu, n_q_heads, n_kv_heads, ctypes.byref(share)))
    return share


def mmsp_zigzag_gather(T, N, row_bytes, seq, shards, stream=0):
    _check(_lib.mmsp_zigzag_gather(T, N, row_bytes, _ptr(seq), _ptr(shards), stream or None))


def mmsp_zigzag_scatter(T, N, row_bytes, shards, seq, stream=0):
    _check(_lib.mmsp_zigzag_scatter(T, N, row_bytes, _ptr(shards), _ptr(seq), stream or None))


def mmsp_a2a_pack_heads(n_tokens, U, slice_bytes, x, y, stream=0):
    _check(_lib.mmsp_a2a_pack_heads(n_tokens, U, slice_bytes, _ptr(x), _ptr(y), stream or None))


def mmsp_a2a_unpack_heads(n_tokens, U, slice_bytes, y, x, stream=0):
    _check(_lib.mmsp_a2a_unpack_heads(n_tokens, U, slice_bytes, _ptr(y), _ptr(x), stream or None))


def mmsp_workspace_bytes(shape, n_q_max, n_k_max, backward):
    return _lib.mmsp_workspace_bytes(ctypes.byref(shape), n_q_max, n_k_max, int(backward))


def mmsp_attn_step_fwd(shape, blk, q, k, v, o, lse, accumulate, workspace=None, workspace_bytes=0, stream=0):
    _check(_lib.mmsp_attn_step_fwd(ctypes.byref(shape), ctypes.byref(blk), _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                   _ptr(lse), int(accumulate), _ptr(workspace), workspace_bytes, stream or None))


def mmsp_attn_merge(shape, row0, n_rows, o_acc, lse_acc, o_part, lse_part, o_final=None, stream=0):
    _check(_lib.mmsp_attn_merge(ctypes.byref(shape), row0, n_rows, _ptr(o_acc), _ptr(lse_acc), _ptr(o_part),
                                _ptr(lse_part), _ptr(o_final), stream or None))


def mmsp_attn_delta(shape, row0, n_rows, o_final, d_o, delta, stream=0):
    _check(_lib.mmsp_attn_delta(ctypes.byref(shape), row0, n_rows, _ptr(o_final), _ptr(d_o), _ptr(delta),
                                stream or None))


def mmsp_attn_step_bwd_static(shape, blk, q, k, v, o_final, d_o, lse_final, delta, compute_delta, dq_acc, dk, dv,
                              accumulate_dkdv, stream=0):
    _check(_lib.mmsp_attn_step_bwd_static(ctypes.byref(shape), ctypes.byref(blk), _ptr(q), _ptr(k), _ptr(v),
                                          _ptr(o_final), _ptr(d_o), _ptr(lse_final), _ptr(delta), int(compute_delta),
                                          _ptr(dq_acc), _ptr(dk), _ptr(dv), int(accumulate_dkdv), stream or None))


def mmsp_attn_step_bwd(shape, blk, q, k, v, o_final, d_o, lse_final, delta, compute_delta, dq_acc, dk, dv,
                       accumulate_dkdv, workspace=None, workspace_bytes=0, stream=0):
    _check(_lib.mmsp_attn_step_bwd(ctypes.byref(shape), ctypes.byref(blk), _ptr(q), _ptr(k), _ptr(v), _ptr(o_final),
                                   _ptr(d_o), _ptr(lse_final), _ptr(delta), int(compute_delta), _ptr(dq_acc),
                                   _ptr(dk), _ptr(dv), int(accumulate_dkdv), _ptr(workspace), workspace_bytes,
                                   stream or None))


# ---- inference: rotary positions, the paged cache ----

def make_heads(data, n_heads, dtype, tok_stride, head_stride):
    return MmspHeads(_ptr(data), n_heads, dtype, tok_stride, head_stride)


def make_cache(k, v, strides, n_pages, page_size, page_table=None, table_stride=0, max_pages=0, n_seqs=0, lengths=None, cu_new=None, n_rows=0, most_new=0):
    """strides = (page, token, head) in elements, of K and of V; most_new: the most new tokens of a sequence, if it is known."""
    return MmspCache(_ptr(k), _ptr(v), strides[0], strides[1], strides[2], n_pages, page_size, _ptr(page_table), table_stride, max_pages, n_seqs,
                     _ptr(lengths), _ptr(cu_new), n_rows, most_new)


def mmsp_rotary_plan(head_dim, theta, sections):
    rotary = MmspRotary()
    _check(_lib.mmsp_rotary_plan(head_dim, theta, len(sections), (_I32 * len(sections))(*sections), ctypes.byref(rotary)))
    return rotary


def _positions(rotary, n_rows, positions, pos_stride):
    """Of a tensor, that it is what the kernel will read: int32, on a GPU, with a position for every row on every axis."""
    if positions is None or positions.__class__ is int:
        return
    if positions.dtype is not sys.modules["torch"].int32 or not positions.is_cuda:
        raise ValueError("positions must be int32 on the GPU, not %s on %s" % (positions.dtype, positions.device))
    last = (rotary.n_axes - 1) * pos_stride + n_rows
    if last > positions.numel() and last > positions.untyped_storage().nbytes() // 4 - positions.storage_offset():
        raise ValueError("positions of %d elements are too few for %d rows on %d axes" % (positions.numel(), n_rows, rotary.n_axes))


def mmsp_rotary_apply(rotary, n_rows, positions, pos_stride, x, y, inverse=False, stream=0):
    """x, y: one or two MmspHeads each."""
    if len(x) != len(y):
        raise ValueError("%d tensors to turn, %d to write" % (len(x), len(y)))
    d = rotary.head_dim
    for h in (*x, *y):
        of = h.of
        if of is not None and (n_rows > of[0] or d > of[1]):
            raise ValueError("a tensor on the GPU with %d rows of head_dim %d is wanted, not %s of %d" % (n_rows, d, "%d" % of[0] if of[0] >= 0 else "one elsewhere", of[1]))
    _positions(rotary, n_rows, positions, pos_stride)
    _check(_lib.mmsp_rotary_apply(ctypes.byref(rotary), n_rows, _ptr(positions), pos_stride, len(x), (MmspHeads * len(x))(*x),
                                  (MmspHeads * len(y))(*y), int(inverse), stream or None))


def mmsp_cache_append(shape, cache, rotary, positions, pos_stride, q, k, v, q_out=None, stream=0):
    if rotary is not None:
        _positions(rotary, cache.n_rows, positions, pos_stride)
    _check(_lib.mmsp_cache_append(ctypes.byref(shape), ctypes.byref(cache), None if rotary is None else ctypes.byref(rotary), _ptr(positions),
                                  pos_stride, _ptr(q), _ptr(k), _ptr(v), _ptr(q_out), stream or None))


def mmsp_cache_workspace_bytes(shape, cache):
    return _lib.mmsp_cache_workspace_bytes(ctypes.byref(shape), ctypes.byref(cache))


def mmsp_cache_attn(shape, cache, q, o_final, o, lse, workspace=None, workspace_bytes=0, stream=0):
    _check(_lib.mmsp_cache_attn(ctypes.byref(shape), ctypes.byref(cache), _ptr(q), _ptr(o_final), _ptr(o), _ptr(lse), _ptr(workspace),
                                workspace_bytes, stream or None))


def mmsp_cache_copy_pages(shape, cache, n_layers, layer_stride, copies, n_copies, stream=0):
    """copies: device int32 tensor [n_copies, 3] of (src, dst, n_tokens)."""
    if copies is not None and not isinstance(copies, int) and (copies.dtype is not sys.modules["torch"].int32 or not copies.is_cuda or not copies.is_contiguous()
                                                              or copies.numel() < 3 * n_copies):
        raise ValueError("copies must be int32 [%d, 3] on the GPU, contiguous, not %s %s on %s" % (n_copies, copies.dtype, tuple(copies.shape), copies.device))
    _check(_lib.mmsp_cache_copy_pages(ctypes.byref(shape), ctypes.byref(cache), n_layers, layer_stride, _ptr(copies), n_copies, stream or None))


def _host(a, kind, dtype, what):
    """Pointer to a numpy array's data; only the very type and layout the call reads is taken."""
    if not isinstance(a, np.ndarray) or a.dtype != dtype or not a.flags.c_contiguous:
        raise ValueError("%s must be a C-contiguous numpy array of %s" % (what, np.dtype(dtype).name))
    return a.ctypes.data_as(ctypes.POINTER(kind))


def make_pages(refs, free_pages, page_size):
    """Bookkeeping in two numpy int32 arrays of n_pages, which the caller keeps."""
    if len(refs) != len(free_pages):
        raise ValueError("refs and free_pages must have one entry for each page")
    pages = MmspPages(len(refs), page_size, _host(refs, _I32, np.int32, "refs"), _host(free_pages, _I32, np.int32, "free_pages"), 0)
    _check(_lib.mmsp_pages_init(ctypes.byref(pages)))
    return pages


def mmsp_pages_grow(pages, row, n_old, n_new):
    """Returns the page copy to make, (src, dst, n_tokens), or None."""
    copy, n = MmspPageCopy(), _I32()
    _check(_lib.mmsp_pages_grow(ctypes.byref(pages), _host(row, _I32, np.int32, "row"), len(row), n_old, n_new, ctypes.byref(copy), ctypes.byref(n)))
    return (copy.src, copy.dst, copy.n_tokens) if n.value else None


def mmsp_pages_fork(pages, row, n_tokens, new_row):
    if len(new_row) < len(row):
        raise ValueError("new_row has %d entries, row %d" % (len(new_row), len(row)))
    _check(_lib.mmsp_pages_fork(ctypes.byref(pages), _host(row, _I32, np.int32, "row"), len(row), n_tokens, _host(new_row, _I32, np.int32, "new_row")))


def mmsp_pages_free(pages, row, n_tokens):
    _check(_lib.mmsp_pages_free(ctypes.byref(pages), _host(row, _I32, np.int32, "row"), len(row), n_tokens))


def mmsp_pages_compact(pages, rows, n_tokens):
    """rows [n_seqs, max_pages], n_tokens [n_seqs] (int64).  Returns (copies [n, 3] int32, pages in use)."""
    if rows.ndim != 2 or len(rows) != len(n_tokens):
        raise ValueError("one row and one length for each sequence")
    copies, n, used = np.zeros((pages.n_pages, 3), dtype=np.int32), _I32(), _I32()
    _check(_lib.mmsp_pages_compact(ctypes.byref(pages), _host(rows, _I32, np.int32, "rows"), rows.shape[1], rows.shape[1], len(rows),
                                   _host(n_tokens, _I64, np.int64, "n_tokens"), copies.ctypes.data_as(_COPY), ctypes.byref(n), ctypes.byref(used)))
    return copies[:n.value], used.value
