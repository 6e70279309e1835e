"""The operators around a paged key-value cache, as a rank's inference (and, for the rotary positions, training) program
calls them: what is measured of them, their plain forms and their values in 64 bits.

Kinds of case
  attn     attention of one or a few new tokens per sequence over a paged cache; `here` is the share of pages that this rank holds
  append   new tokens: Q and K rotated, K and V written into the cache's pages
  rotary   rotary positions with 1 to 3 axes (time, height, width) of Q and K, or of their gradients (`inverse`)
  pages    page copies over all layers: `fork` (the partly filled last pages of forked sequences) or `compact` (whole pages)
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
THETA = 1e6


def listed():
    return [
        # The first answer token on a question of some two hundred tokens: the smallest call, a chain of latencies.
        dict(name="attn_one_short", kind="attn", dtype="bf16", hq=28, hkv=4, d=128, seqs=1, longest=203, shortest=203, new=1, page=16, here=1.0, order="heads", mix=1),
        # One answer on a 256K-token video: four KV heads, the work of the chip cut along the cache's length.
        dict(name="attn_one_256k", kind="attn", dtype="bf16", hq=28, hkv=4, d=128, seqs=1, longest=262144, shortest=262144, new=1, page=64, here=1.0, order="heads", mix=2),
        # A batch of answers on clips and videos of very different lengths.
        dict(name="attn_batch_ragged", kind="attn", dtype="bf16", hq=28, hkv=4, d=128, seqs=64, longest=16384, shortest=150, new=1, page=16, here=1.0, order="heads", mix=3),
        # Short drafts being verified, up to five tokens a sequence, some sequences pausing; pages of 48 end inside tiles.
        dict(name="attn_draft", kind="attn", dtype="bf16", hq=28, hkv=4, d=128, seqs=16, longest=5003, shortest=40, new=5, page=48, here=1.0, order="tokens", mix=4),
        # One head share and an eighth of the pages of a 256K-token sequence: what a rank of a mesh adds to the joined result.
        dict(name="attn_share", kind="attn", dtype="bf16", hq=7, hkv=1, d=128, seqs=2, longest=200003, shortest=131072, new=1, page=128, here=0.125, order="heads", mix=5),
        # The full-precision configuration that the parity work runs on.
        dict(name="attn_f32_small", kind="attn", dtype="f32", hq=2, hkv=1, d=64, seqs=5, longest=1001, shortest=1, new=2, page=16, here=1.0, order="tokens", mix=6),
        # A decode step's rows for a batch of 64.
        dict(name="append_64", kind="append", dtype="bf16", hq=28, hkv=4, d=128, seqs=64, longest=4096, shortest=100, new=1, page=16, axes=3, order="heads", mix=7),
        # Prompts of some frames and text written after their prefill.
        dict(name="append_prompts", kind="append", dtype="bf16", hq=28, hkv=4, d=128, seqs=5, longest=8011, shortest=700, new=8011, page=64, axes=3, order="heads", mix=8),
        # Q and K of a rank's 8192 rows of the 256K-token workload, slices of one projection.
        dict(name="rotary_8k", kind="rotary", dtype="bf16", out="bf16", hq=28, hkv=4, d=128, rows=8192, axes=3, inverse=False, fused=True),
        # Their gradients, as the backward leaves them, on the way to the projection's backward.
        dict(name="rotary_8k_gradient", kind="rotary", dtype="f32", out="bf16", hq=28, hkv=4, d=128, rows=8192, axes=3, inverse=True, fused=False),
        # Eight continuations of one video: the partly filled last page, in all layers.
        dict(name="pages_fork", kind="pages", what="fork", dtype="bf16", hkv=4, d=128, layers=28, pages=300, page=16, copies=8, order="heads", mix=9),
        # A cache moved to the front of its pool.
        dict(name="pages_compact", kind="pages", what="compact", dtype="bf16", hkv=4, d=128, layers=28, pages=1003, page=64, copies=301, order="heads", mix=10),
    ]


_MOST_BYTES = 2.0e9                     # the largest listed case moves 2.2e9


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn", "append", "append", "rotary", "rotary", "pages"])
    while True:
        f32 = rng.random() < 0.2
        hq, hkv = rng.choice([(2, 1), (4, 2), (8, 8)]) if f32 else rng.choice([(28, 4), (28, 4), (14, 2), (7, 1), (4, 2), (8, 8)])
        case = dict(kind=kind, dtype="f32" if f32 else "bf16", hq=hq, hkv=hkv, d=rng.choice([64, 128]) if f32 else 128)
        if kind == "attn":
            seqs = _log_int(rng, 1, 200)
            longest = _log_int(rng, 20, 262144)
            case.update(seqs=seqs, longest=longest, shortest=_log_int(rng, 1, longest), new=rng.choice([1, 1, 1, rng.randint(2, 16)]),
                        page=16 * rng.choice([1, 1, 2, 3, 4, 8, 16]), here=rng.choice([1.0, 1.0, 1.0, 0.5, 0.125]),
                        order=rng.choice(["heads", "heads", "tokens"]), mix=rng.randrange(1 << 20))
            if seqs * longest * hkv > 6 << 20:          # the plain form pads every sequence to the longest
                continue
        elif kind == "append":
            seqs, longest = _log_int(rng, 1, 200), _log_int(rng, 20, 16384)
            case.update(seqs=seqs, longest=longest, shortest=_log_int(rng, 1, longest), new=rng.choice([1, 1, rng.randint(2, 16), longest]),
                        page=16 * rng.choice([1, 1, 2, 3, 4, 8, 16]), axes=rng.choice([1, 3, 3]), order=rng.choice(["heads", "heads", "tokens"]),
                        mix=rng.randrange(1 << 20))
            if seqs * longest > 1 << 19:
                continue
        elif kind == "rotary":
            inverse = rng.random() < 0.5
            case.update(rows=_log_int(rng, 1, 40000), axes=rng.choice([1, 2, 3, 3]), inverse=inverse, fused=rng.random() < 0.5)
            case["out"] = case["dtype"]
            if inverse and not f32 and rng.random() < 0.7:
                case["dtype"] = "f32"
        else:
            del case["hq"]
            pages = _log_int(rng, 20, 4000)
            case.update(what=rng.choice(["fork", "compact"]), layers=rng.choice([1, 4, 28]), pages=pages, page=16 * rng.choice([1, 1, 2, 3, 4, 8]),
                        copies=rng.randint(1, max(1, pages // 3)), order=rng.choice(["heads", "heads", "tokens"]), mix=rng.randrange(1 << 20))
            if pages * case["page"] * case["layers"] * hkv * case["d"] * 4 > 6e9:
                continue
        if work(case)["bytes"] <= _MOST_BYTES:
            return case


# ---- sizes that a case stands for -----------------------------------------------------------------

def _elt(name):
    return 4 if name == "f32" else 2


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _lengths(case):
    """(tokens of each sequence with its new ones, new tokens of each), numpy."""
    r = np.random.RandomState(case["mix"])
    n = np.exp(r.uniform(math.log(case["shortest"]), math.log(case["longest"]), case["seqs"])).round().astype(np.int64)
    n[0], n[-1] = case["longest"], (case["longest"] if case["seqs"] == 1 else case["shortest"])
    new = np.ones_like(n)
    if case["new"] > 16:                                # whole prompts
        new = n.copy()
    elif case["new"] > 1:
        new = np.minimum(n, r.randint(0, case["new"] + 1, case["seqs"]))
        new[0] = min(n[0], case["new"])
    return n, new


def _held(case):
    """The page table, numpy int32 [seqs, pages of the longest + 1]: pages in random order, -1 where there is none or it lies on another rank; and the pool's size."""
    n, _ = _lengths(case)
    r = np.random.RandomState(case["mix"] + 1)
    used = -(-n // case["page"])
    table = np.full((case["seqs"], int(used.max()) + 1), -1, dtype=np.int32)
    have = (np.arange(table.shape[1])[None, :] < used[:, None]) & (r.random_sample(table.shape) < case.get("here", 1.0))
    count = int(have.sum())
    pool = count + max(3, count // 16)
    table[have] = r.permutation(pool)[:count]
    return table, pool


def _seen(case):
    """Pairs of a new token and a cache token that it sees on this rank, and cache tokens here that any new one sees."""
    n, new = _lengths(case)
    table, _ = _held(case)
    held = np.zeros((table.shape[0], table.shape[1] * case["page"] + 1), dtype=np.int64)
    held[:, 1:] = np.cumsum(np.repeat(table >= 0, case["page"], axis=1), axis=1)
    row = np.repeat(np.arange(len(n)), new)
    first = np.concatenate([[0], np.cumsum(new)])
    at = n[row] - new[row] + np.arange(len(row)) - first[row]
    return int(held[row, at + 1].sum()), int(held[np.arange(len(n)), n][new > 0].sum())


def _copies(case):
    """Page copies (source, target, tokens), numpy int32 [copies, 3]: targets differ from each other and from every source."""
    r = np.random.RandomState(case["mix"])
    p, c = case["pages"], case["copies"]
    order = r.permutation(p)
    if case["what"] == "compact":                       # holes at the front, pages in use behind them
        order = np.concatenate([r.permutation(p // 2), p // 2 + r.permutation(p - p // 2)])
        return np.stack([order[p // 2:p // 2 + c], order[:c], np.full(c, case["page"])], 1).astype(np.int32)
    return np.stack([order[c + r.randint(0, max(1, min(p - c, c // 4)), c)], order[:c], r.randint(1, case["page"], c)], 1).astype(np.int32)


def _sections(case):
    half = case["d"] // 2
    return {1: [half], 2: [half // 2, half - half // 2], 3: [half // 4, 3 * half // 8, 3 * half // 8]}[case["axes"]]


def work(case):
    kind = case["kind"]
    if kind == "pages":
        tokens = int(_copies(case)[:, 2].sum())
        return {"bytes": 4 * case["layers"] * tokens * case["hkv"] * case["d"] * _elt(case["dtype"]) + 12 * case["copies"], "flops": 0}
    hq, hkv, d, e = case["hq"], case["hkv"], case["d"], _elt(case["dtype"])
    if kind == "rotary":
        elems = case["rows"] * (hq + hkv) * d
        return {"bytes": elems * (e + _elt(case["out"])) + 4 * case["axes"] * case["rows"], "flops": 3 * elems}
    n, new = _lengths(case)
    rows = int(new.sum())
    table = 4 * (int((-(-n // case["page"]))[new > 0].sum()) if kind == "attn" else rows) + 8 * case["seqs"]
    if kind == "append":
        return {"bytes": 2 * rows * (hq + 2 * hkv) * d * e + 4 * case["axes"] * rows + table, "flops": 3 * rows * (hq + hkv) * d}
    pairs, tokens = _seen(case)
    return {"bytes": tokens * hkv * 2 * d * e + 2 * rows * hq * d * e + 4 * rows * hq + table, "flops": 4 * d * hq * pairs}


# ---- inputs -----------------------------------------------------------------------------------------

def _maker(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*size, dtype=torch.float32, sigma=1.0):
        x = torch.empty(size, dtype=dtype, device=DEV)
        return x.normal_(0.0, sigma, generator=gen)
    return normal


def _pool(case, normal, pages, *front):
    """K and V of a pool as [*front, pages, heads, page, d]; order `tokens`: a page holds its tokens one after the other, all heads of each."""
    size = (*front, pages, case["hkv"], case["page"], case["d"])
    if case["order"] == "heads":
        return [normal(*size, dtype=_dtype(case["dtype"])) for _ in range(2)]
    size = (*front, pages, case["page"], case["hkv"], case["d"])
    return [normal(*size, dtype=_dtype(case["dtype"])).transpose(-2, -3) for _ in range(2)]


def _positions(case, rows, seed):
    """int32 [axes, rows]: frames of 14 x 14 tokens one after the other, from a place in a long video on."""
    start = 1 + seed % 100003
    r = torch.arange(rows, device=DEV)
    if case["axes"] == 1:
        p = (start + r)[None]
    else:
        p = torch.stack([start + r // 196, start + r % 196 // 14, start + r % 14])[:case["axes"]]
    return p.to(torch.int32).contiguous()


def _cu(new):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)


def prepare(case, seed):
    kind, s, normal = case["kind"], {"case": case}, _maker(seed)
    if kind == "pages":
        s["k"], s["v"] = _pool(case, normal, case["pages"], case["layers"])
        s["copies"] = torch.from_numpy(_copies(case)).to(DEV)
        return s
    hq, hkv, d, dtype = case["hq"], case["hkv"], case["d"], _dtype(case["dtype"])
    if kind == "rotary":
        rows = case["rows"]
        if case["fused"]:                               # slices of one projection's output
            x = normal(rows, hq + 2 * hkv, d, dtype=dtype)
            s["q"], s["k"] = x[:, :hq], x[:, hq:hq + hkv]
        else:
            s["q"], s["k"] = normal(rows, hq, d, dtype=dtype), normal(rows, hkv, d, dtype=dtype)
        s["positions"] = _positions(case, rows, seed)
        s["q_out"], s["k_out"] = (torch.empty(rows, h, d, dtype=_dtype(case["out"]), device=DEV) for h in (hq, hkv))
        return s
    n, new = _lengths(case)
    table, pool = _held(case)
    rows = int(new.sum())
    s["page_table"], s["lengths"] = torch.from_numpy(table).to(DEV), torch.from_numpy(n.astype(np.int32)).to(DEV)
    s["cu_new"] = None if case["new"] == 1 else _cu(new)
    s["k_pool"], s["v_pool"] = _pool(case, normal, pool)
    s["scale"] = 1.0 / math.sqrt(d)
    if kind == "append":
        x = normal(rows, hq + 2 * hkv, d, dtype=dtype)
        s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        s["positions"] = _positions(case, rows, seed)
        s["q_out"] = torch.empty(rows, hq, d, dtype=dtype, device=DEV)
        return s
    s["q"] = normal(rows, hq, d, dtype=dtype)
    s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(hq, rows, dtype=torch.float32, device=DEV)
    s["most_new"] = int(new.max())
    return s


# ---- plain forms --------------------------------------------------------------------------------------

def _angles(case, positions):
    """cos and sin [rows, 1, d / 2] of every pair's angle, taken in 64 bits: a far position times a frequency keeps few of 24 bits behind the point."""
    half = case["d"] // 2
    axis = torch.repeat_interleave(torch.arange(case["axes"], device=DEV), torch.tensor(_sections(case), device=DEV), output_size=half)
    freq = THETA ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    a = positions.double()[axis].T * freq
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _turned(x, cos, sin):
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_rotary(s):
    cos, sin = _angles(s["case"], s["positions"])
    if s["case"]["inverse"]:
        sin = -sin
    return [_turned(x, cos, sin).to(y.dtype) for x, y in ((s["q"], s["q_out"]), (s["k"], s["k_out"]))]


def _row_places(s, rows):
    """Of every row: its sequence, its number among that one's new tokens, its place in the cache."""
    r = torch.arange(rows, device=DEV)
    if s["cu_new"] is None:
        return r, torch.zeros_like(r), s["lengths"].long() - 1
    cu = s["cu_new"].long()
    seq = torch.searchsorted(cu, r, right=True) - 1
    i = r - cu[seq]
    return seq, i, s["lengths"].long()[seq] - (cu[seq + 1] - cu[seq]) + i


def _plain_append(s):
    case = s["case"]
    cos, sin = _angles(case, s["positions"])
    seq, _, at = _row_places(s, s["q"].shape[0])
    page = s["page_table"][seq, at // case["page"]].long()
    s["k_pool"][page, :, at % case["page"]] = _turned(s["k"], cos, sin).to(s["k"].dtype)
    s["v_pool"][page, :, at % case["page"]] = s["v"]
    return _turned(s["q"], cos, sin).to(s["q"].dtype), s["k_pool"], s["v_pool"]


def _plain_attn(s):
    case, q = s["case"], s["q"]
    rows, hq, d = q.shape
    hkv, p, seqs, new = case["hkv"], case["page"], case["seqs"], s["most_new"]
    seq, i, at = _row_places(s, rows)
    j = torch.arange(case["longest"], device=DEV)
    page = s["page_table"][:, j // p].long()                                  # [seqs, tokens]
    k, v = (x.transpose(1, 2)[page.clamp(min=0), j % p].float() for x in (s["k_pool"], s["v_pool"]))   # [seqs, tokens, hkv, d]
    padded = torch.zeros(seqs, new, hq, d, device=DEV)
    padded[seq, i] = q.float()
    last = torch.full((seqs, new), -1, device=DEV)
    last[seq, i] = at
    x = padded.view(seqs, new, hkv, hq // hkv, d).transpose(1, 2).reshape(seqs, hkv, -1, d)
    score = torch.matmul(x, k.permute(0, 2, 3, 1).contiguous()) * s["scale"]  # [seqs, hkv, new * group, tokens]
    seen = (j <= last[:, :, None]) & (page >= 0)[:, None]
    score = score.view(seqs, hkv, new, hq // hkv, -1).masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(seqs, hkv, -1, len(j)), v.transpose(1, 2).contiguous()).view(seqs, hkv, new, hq // hkv, d)
    o = torch.where(total > 0, o / total, 0.0).transpose(1, 2).reshape(seqs, new, hq, d)
    lse = (top + torch.log(total)).transpose(1, 2).reshape(seqs, new, hq)
    return o[seq, i].to(q.dtype), lse[seq, i].T.contiguous()


def _plain_pages(s):
    src, dst, count = s["copies"].long().unbind(1)
    copied = (torch.arange(s["case"]["page"], device=DEV) < count[:, None])[:, None, :, None]
    s["k"][:, dst] = torch.where(copied, s["k"][:, src], s["k"][:, dst])
    s["v"][:, dst] = torch.where(copied, s["v"][:, src], s["v"][:, dst])
    return s["k"], s["v"]


# ---- the framework's calls ------------------------------------------------------------------------------

def _handle(s):
    """The descriptors and the workspace that a program makes once for buffers that it keeps."""
    from paper_2408_10188_amd import binding as B
    from paper_2408_10188_amd import paged, ring
    case, h = s["case"], {"B": B}
    io = B.MMSP_F32 if case["dtype"] == "f32" else B.MMSP_BF16
    if "axes" in case:
        h["rotary"] = B.mmsp_rotary_plan(case["d"], THETA, _sections(case))
    if case["kind"] == "rotary":
        h["x"], h["y"] = [paged.heads_of(s["q"]), paged.heads_of(s["k"])], [paged.heads_of(s["q_out"]), paged.heads_of(s["k_out"])]
    elif case["kind"] == "pages":
        h["shape"], h["cache"] = paged.shape_for(s["k"][0], io), paged.cache_for(s["k"][0], s["v"][0])
    else:
        rows = s["q"].shape[0]
        h["shape"] = ring.shape_for(s["q"], s.get("k", s["q"][:, :case["hkv"]]), io, rows, s["scale"])
        h["cache"] = paged.cache_for(s["k_pool"], s["v_pool"], s["page_table"], s["lengths"], rows, s["cu_new"])
        if case["kind"] == "attn":
            h["room"] = B.mmsp_cache_workspace_bytes(h["shape"], h["cache"])
            h["ws"] = torch.empty(max(h["room"], 16), dtype=torch.uint8, device=DEV)
    s["handle"] = h
    return h


def _own(s):
    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    h = s.get("handle") or _handle(s)
    B, kind = h["B"], case["kind"]
    if kind == "attn":
        B.mmsp_cache_attn(h["shape"], h["cache"], s["q"], s["o"], None, s["lse"], h["ws"], h["room"], stream)
        return s["o"], s["lse"]
    if kind == "append":
        B.mmsp_cache_append(h["shape"], h["cache"], h["rotary"], s["positions"], s["positions"].shape[1], s["q"], s["k"], s["v"], s["q_out"], stream)
        return s["q_out"], s["k_pool"], s["v_pool"]
    if kind == "rotary":
        B.mmsp_rotary_apply(h["rotary"], case["rows"], s["positions"], s["positions"].shape[1], h["x"], h["y"], case["inverse"], stream)
        return s["q_out"], s["k_out"]
    B.mmsp_cache_copy_pages(h["shape"], h["cache"], case["layers"], s["k"].stride(0), s["copies"], case["copies"], stream)
    return s["k"], s["v"]


def run(state):
    if own:
        return _own(state)
    return {"attn": _plain_attn, "append": _plain_append, "rotary": _plain_rotary, "pages": _plain_pages}[state["case"]["kind"]](state)


# ---- the same in 64 bits ----------------------------------------------------------------------------------

def _exact_turn(x, case, positions, sign):
    """Each pair as a complex number, times e^(i angle)."""
    half = case["d"] // 2
    y = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    pair = 0
    for axis, count in enumerate(_sections(case)):
        for i in range(pair, pair + count):
            z = torch.polar(torch.ones_like(positions[axis], dtype=torch.float64), sign * positions[axis].double() * THETA ** (-2.0 * i / case["d"]))
            w = torch.complex(x[..., i].double(), x[..., i + half].double()) * z[:, None]
            y[..., i], y[..., i + half] = w.real, w.imag
        pair += count
    return y


def _exact_attn(case, s):
    n, new = _lengths(case)
    table, _ = _held(case)
    hkv, p = case["hkv"], case["page"]
    group = case["hq"] // hkv
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    row = 0
    for b in range(case["seqs"]):
        held = [c for c in range(-(-int(n[b]) // p)) if table[b, c] >= 0]
        pages = torch.tensor([int(table[b, c]) for c in held], dtype=torch.long, device=DEV)
        at = (torch.tensor(held, dtype=torch.long, device=DEV)[:, None] * p + torch.arange(p, device=DEV)).reshape(-1)
        rows = slice(row, row + int(new[b]))
        row += int(new[b])
        if new[b] == 0 or not held:
            continue
        own_at = torch.arange(int(n[b] - new[b]), int(n[b]), device=DEV)
        hidden = at > own_at[:, None]
        for h in range(hkv):
            k, v = (x[pages, h].reshape(-1, case["d"]).double() for x in (s["k_pool"], s["v_pool"]))
            heads = slice(h * group, (h + 1) * group)
            x = s["q"][rows, heads].double()                                    # [new, group, d]
            score = (x.reshape(-1, case["d"]) @ k.T * s["scale"]).view(x.shape[0], group, -1).masked_fill(hidden[:, None], -math.inf)
            total = torch.logsumexp(score, -1)
            weight = torch.exp(score - torch.where(total == -math.inf, 0.0, total)[..., None])
            o[rows, heads] = (weight.reshape(-1, len(at)) @ v).view(x.shape)
            lse[heads, rows] = total.T
    return o, lse


def exact(case, seed):
    if case["kind"] == "pages":
        return None
    s = prepare(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(case, s)
    if case["kind"] == "rotary":
        sign = -1.0 if case["inverse"] else 1.0
        return [_exact_turn(s[x], case, s["positions"], sign) for x in ("q", "k")]
    n, new = _lengths(case)
    table, _ = _held(case)
    k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
    k, row = _exact_turn(s["k"], case, s["positions"], 1.0), 0
    for b in range(case["seqs"]):
        at = np.arange(n[b] - new[b], n[b])
        page, slot = (torch.from_numpy(x.astype(np.int64)).to(DEV) for x in (table[b, at // case["page"]], at % case["page"]))
        k_pool[page, :, slot] = k[row:row + len(at)]
        v_pool[page, :, slot] = s["v"][row:row + len(at)].double()
        row += len(at)
    return _exact_turn(s["q"], case, s["positions"], 1.0), k_pool, v_pool
