"""Operators of a serving loop over a paged key/value cache (include/loopspec.h).

For one layer and one step of a batch:

    cache = PagedCache(k, v)                     # [n_pages, n_kv_heads, page_size, head_dim], any strides
    batch = Batch(seq_len, table, prefix_len=P, prefix_table=prefix)
    q = rope_append(q, k_new, v_new, cache, batch, rope_frequencies(head_dim))
    o = prefix_attention(q, cache, batch)        # every sequence behind the same prefix
    ...
    tokens, probs, kept = sample(logits, u, temperature, top_k, top_p, min_p)

For long contexts the cache may be a QuantizedCache (8-bit pages), attention window_attention (a window and a few first
positions, or all, over either cache), and between steps

    seq_len, table, refs, short = fork_pages(seq_len, table, parent, refs, caches, P, window, sinks, room=1)

continues some rows, several times or not at all, and lets their pages go that nobody needs.

Argument marshalling only: the work runs in the HIP library, on the current
stream of the tensors' device, without waiting for it, and records no
gradients.  Wrong shapes, types or
devices raise ValueError, what the library refuses raises LoopSpecError.
"""
from __future__ import annotations

import ctypes
import math
import operator
from typing import Optional

from . import binding as B

_DTYPES = None


def _dtype(t) -> int:
    global _DTYPES
    if _DTYPES is None:
        import torch
        _DTYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16, torch.float16: B.F16}
    return _DTYPES.get(t.dtype, -1)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _size(n: int, what: str) -> int:
    """A size for a 32-bit field, which would keep the low bits of a larger one."""
    if not 0 <= n < 1 << 31:
        raise ValueError(f"{what}: {n} is not in [0, 2^31)")
    return n


def _whole(n, what: str) -> int:
    n = operator.index(n)
    _need(n >= 0, f"{what}: not below zero")
    return n


def _ints(t, shape, device, what: str):
    import torch
    if not (t.dtype is torch.int32 and t.device == device and t.dim() == len(shape) and t.stride(-1) == 1
            and shape[0] in (None, t.shape[0]) and shape[-1] in (None, t.shape[-1])):
        raise ValueError(f"{what}: int32, unit stride, shape {list(shape)} on {device}")
    return t.data_ptr()


def _launch(device, call, *args) -> int:
    """One call of the library on the device's current stream."""
    import torch
    stream = torch._C._cuda_getCurrentRawStream(device.index)   # torch.cuda.current_stream without its object, 2 us
    if torch._C._cuda_getDevice() == device.index:
        return call(*args, stream)
    with torch.cuda.device(device):
        return call(*args, stream)


def _check(rc: int, name: str) -> None:
    if rc:
        raise B.LoopSpecError(rc, f"{name} refused its arguments" if rc == B.EINVAL else f"{name} failed")


class PagedCache:
    """Pages of keys and values: two fp16 or bf16 tensors [n_pages, n_kv_heads, page_size, head_dim] on one device.
    The last stride is 1 and the others multiples of 8, so a cache that stores positions before heads comes as a
    transposed view.  page_size is a multiple of 16; head_dim 16, 32, 64, 96 or 128."""

    def __init__(self, k, v):
        _need(k.dim() == 4 and k.shape == v.shape, "keys and values: [n_pages, n_kv_heads, page_size, head_dim] alike")
        _need(k.dtype == v.dtype and _dtype(k) in (B.BF16, B.F16), "keys and values: both bfloat16 or both float16")
        _need(k.is_cuda and k.device == v.device, "keys and values: on one GPU")
        _need(k.stride(3) == 1 and v.stride(3) == 1, "keys and values: elements of a head next to each other")
        self.k, self.v, self.device, self.dtype = k, v, k.device, k.dtype
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = (_size(n, "keys and values") for n in k.shape)
        self._c = B.PagedCacheC(_dtype(k), self.n_pages, self.page_size, self.n_kv_heads, self.head_dim, k.data_ptr(),
                                v.data_ptr(), *k.stride()[:3], *v.stride()[:3])
        self._ref = ctypes.byref(self._c)
        self._raw = bytes(self._c), bytes(ctypes.sizeof(B.PageScalesC))         # (for lists of caches; no scales)

    _scales_ref = None

    def _for(self, dtype):
        return self._ref


class QuantizedCache:
    """Pages of keys and values in 8 bits: float8_e4m3fn codes k, v [n_pages, n_kv_heads, page_size, head_dim] and
    float8_e8m0fnu scales k_scale, v_scale [n_pages, n_kv_heads, page_size / 16], one for 16 positions of a head; an
    element stands for code * scale.  The last strides are 1, the codes' others multiples of 16.  Sizes as in PagedCache;
    queries are float16 or bfloat16.  Scales of pages that hold nothing yet do not matter."""

    dtype = None                              # (the queries' decides)

    def __init__(self, k, v, k_scale, v_scale):
        import torch
        _need(k.dim() == 4 and k.shape == v.shape, "keys and values: [n_pages, n_kv_heads, page_size, head_dim] alike")
        _need(k.dtype == v.dtype == torch.float8_e4m3fn, "keys and values: float8_e4m3fn")
        _need(k_scale.dtype == v_scale.dtype == torch.float8_e8m0fnu, "scales: float8_e8m0fnu")
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = (_size(n, "keys and values") for n in k.shape)
        blocks = (self.n_pages, self.n_kv_heads, self.page_size // 16)
        _need(k_scale.shape == v_scale.shape == blocks, "scales: [n_pages, n_kv_heads, page_size / 16]")
        _need(k.is_cuda and k.device == v.device == k_scale.device == v_scale.device, "keys, values and scales: on one GPU")
        _need(k.stride(3) == 1 and v.stride(3) == 1, "keys and values: elements of a head next to each other")
        _need(blocks[2] < 2 or k_scale.stride(2) == v_scale.stride(2) == 1, "scales: those of a page next to each other")
        self.k, self.v, self.k_scale, self.v_scale, self.device = k, v, k_scale, v_scale, k.device
        self._scales = B.PageScalesC(k_scale.data_ptr(), v_scale.data_ptr(), *k_scale.stride()[:2], *v_scale.stride()[:2])
        self._scales_ref = ctypes.byref(self._scales)
        self._by_type = {t: B.PagedCacheC(d, *k.shape[:1], self.page_size, self.n_kv_heads, self.head_dim, k.data_ptr(),
                                          v.data_ptr(), *k.stride()[:3], *v.stride()[:3])
                         for t, d in ((torch.float16, B.F16), (torch.bfloat16, B.BF16))}
        self._raw = bytes(self._by_type[torch.float16]), bytes(self._scales)

    def _for(self, dtype):
        if dtype not in self._by_type:
            raise ValueError("queries of an 8-bit cache: float16 or bfloat16")
        return ctypes.byref(self._by_type[dtype])


class Batch:
    """The sequences of a step.  seq_len [n]: own positions of each, with this step's tokens; table [n, pages]: their
    pages; q_start [n + 1] (ascending): first token of each, None when every sequence has one.  All int32 on the GPU,
    read when the kernels run (change them in place).  prefix_len positions in the pages prefix_table come before every sequence's own.
    Tokens outside q_start's range and those of a sequence with seq_len < 0 are padding."""

    def __init__(self, seq_len, table, q_start=None, prefix_len: int = 0, prefix_table=None):
        n, dev = seq_len.shape[0], seq_len.device
        _need(seq_len.is_cuda, "seq_len: on the GPU")
        self.seq_len, self.table, self.q_start, self.prefix_table = seq_len, table, q_start, prefix_table
        self.n_seqs, self.prefix_len, self.device = _size(n, "seq_len"), _size(int(prefix_len), "prefix_len"), dev
        self._c = B.PagedBatchC(n, 0, None if q_start is None else _ints(q_start, (n + 1,), dev, "q_start"),
                                _ints(seq_len, (n,), dev, "seq_len"), _ints(table, (n, None), dev, "table"),
                                table.stride(0), _size(table.shape[1], "table"), self.prefix_len,
                                None if prefix_table is None else _ints(prefix_table, (None,), dev, "prefix_table"))

    def _with(self, tokens: int, cache: PagedCache):
        if self.device != cache.device:
            raise ValueError("batch and cache: on one device")
        c = B.PagedBatchC.from_buffer_copy(self._c)      # a call's own: threads may share the batch
        c.n_tokens = tokens
        return ctypes.byref(c)


def rope_frequencies(rot_dim: int, base: float = 1e4, device="cuda:0"):
    """Radians per position of the rot_dim / 2 pairs: base ** (-2 j / rot_dim), float64."""
    import torch
    return base ** (-torch.arange(rot_dim // 2, dtype=torch.float64, device=device) * 2 / rot_dim)


def _rows(t, heads: int, cache, tokens: int, what: str, dtype):
    if not (t.shape == (tokens, heads, cache.head_dim) and t.dtype is dtype and t.device == cache.device
            and t.stride(2) == 1):
        raise ValueError(f"{what}: [tokens, heads, head_dim] of the cache's type and device, elements adjacent")


def _heads(q, cache):
    """(tokens, heads) of the queries."""
    if q.dim() != 3:
        raise ValueError("q: [tokens, heads, head_dim]")
    tokens, heads, _ = q.shape
    _rows(q, heads, cache, _size(tokens, "q"), "q", cache.dtype or q.dtype)
    return tokens, _size(heads, "q")


def _like(q):
    import torch
    return torch.empty_like(q, memory_format=torch.contiguous_format)


def rope_append(q, k, v, cache, batch: Batch, freq=None, q_norm=None, k_norm=None, eps: float = 1e-6, out=None):
    """Normalise (optional gains q_norm, k_norm: float32 [head_dim]) and rotate the queries and keys of a step's
    tokens, and append keys and values to their sequences' pages.  q [tokens, n_heads, head_dim], k and v [tokens,
    n_kv_heads, head_dim] (views of a fused projection are fine); freq float64 [rot_dim / 2] radians per position
    (None: no rotation), the first rot_dim elements of a head being rotated in halves.  Returns the queries: `out`
    (which may be q) or a new tensor, whose padding rows are then undefined.  Into a QuantizedCache keys and values go
    as codes: a block of 16 positions has the power of two that holds its largest magnitude within 448, and keeps the
    one of positions it holds already where that is larger.  No two sequences may append to one page."""
    import torch
    tokens, heads = _heads(q, cache)
    _rows(k, cache.n_kv_heads, cache, tokens, "k", q.dtype)
    _rows(v, cache.n_kv_heads, cache, tokens, "v", q.dtype)
    if out is None:
        out = _like(q)
    else:
        _rows(out, heads, cache, tokens, "out", q.dtype)
    rot = 0
    if freq is not None:
        _need(freq.dtype == torch.float64 and freq.dim() == 1 and freq.is_contiguous() and freq.device == cache.device,
              "freq: float64 [rot_dim / 2] on the cache's device")
        rot = 2 * freq.shape[0]
    for g in (q_norm, k_norm):
        if g is not None:
            _need(g.dtype == torch.float32 and g.shape == (cache.head_dim,) and g.is_contiguous()
                  and g.device == cache.device, "q_norm, k_norm: float32 [head_dim] on the cache's device")
    a = B.RopeArgs(heads, rot, eps, q.data_ptr(), k.data_ptr(), v.data_ptr(), q.stride(0), q.stride(1),
                   k.stride(0), k.stride(1), v.stride(0), v.stride(1), out.data_ptr(), out.stride(0), out.stride(1),
                   None if freq is None else freq.data_ptr(), None if q_norm is None else q_norm.data_ptr(),
                   None if k_norm is None else k_norm.data_ptr())
    L, ref, more = B.load_library(), batch._with(tokens, cache), ctypes.byref(a)
    if cache._scales_ref is None:
        _check(_launch(cache.device, L.loopspec_rope_append, cache._ref, ref, more), "loopspec_rope_append")
    else:
        _check(_launch(cache.device, L.loopspec_rope_append_quantized, cache._for(q.dtype), cache._scales_ref, ref, more),
               "loopspec_rope_append_quantized")
    return out


def _prefix_held(cache, batch: Batch):
    if batch.prefix_len and (batch.prefix_table is None
                             or batch.prefix_table.shape[0] * cache.page_size < batch.prefix_len):
        raise ValueError("prefix_table: a page for every page_size positions of the prefix")


def prefix_attention(q, cache: PagedCache, batch: Batch, scale: Optional[float] = None, out=None,
                     return_lse: bool = False):
    """Attention of a step's queries [tokens, n_heads, head_dim]: each sees the prefix that all sequences share and its
    own sequence's positions up to its own.  scale defaults to head_dim ** -0.5.  Returns the output (`out`, or a new
    tensor whose padding rows are undefined), with return_lse also the log of each row's sum of exp(score) (float32
    [tokens, n_heads])."""
    import torch
    _need(isinstance(cache, PagedCache), "prefix_attention: 16-bit pages (window_attention takes both)")
    tokens, heads = _heads(q, cache)
    if out is None:
        out = _like(q)
    else:
        _rows(out, heads, cache, tokens, "out", q.dtype)
    lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device) if return_lse else None
    _prefix_held(cache, batch)
    L, ref = B.load_library(), batch._with(tokens, cache)
    nbytes = L.loopspec_prefix_attention_workspace_bytes(cache._ref, ref, heads)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    a = B.AttentionArgs(heads, 1.0 / math.sqrt(cache.head_dim) if scale is None else scale, q.data_ptr(), q.stride(0),
                        q.stride(1), out.data_ptr(), out.stride(0), out.stride(1),
                        None if lse is None else lse.data_ptr())
    _check(_launch(cache.device, L.loopspec_prefix_attention, cache._ref, ref, ctypes.byref(a), ws.data_ptr(), nbytes),
           "loopspec_prefix_attention")
    return (out, lse) if return_lse else out


def window_attention(q, cache, batch: Batch, window: int = 0, sinks: int = 0, scale: Optional[float] = None, out=None,
                     return_lse: bool = False):
    """Attention of a step's queries [tokens, n_heads, head_dim] over 16-bit or 8-bit pages.  The token at position p
    (counted through the prefix) sees the positions j <= p with p - j < window or j < sinks; window 0: all of them.
    Arguments and results as in prefix_attention; a token before its sequence's first position gives zeros."""
    import torch
    tokens, heads = _heads(q, cache)
    if out is None:
        out = _like(q)
    else:
        _rows(out, heads, cache, tokens, "out", q.dtype)
    lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device) if return_lse else None
    _prefix_held(cache, batch)
    # (a window or sinks beyond all positions are those of all positions)
    window, sinks = min(_whole(window, "window"), 1 << 30), min(_whole(sinks, "sinks"), 1 << 30)
    L, ref, c = B.load_library(), batch._with(tokens, cache), cache._for(q.dtype)
    nbytes = L.loopspec_window_attention_workspace_bytes(c, cache._scales_ref, ref, heads, window, sinks)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device) if nbytes else None
    a = B.AttentionArgs(heads, 1.0 / math.sqrt(cache.head_dim) if scale is None else scale, q.data_ptr(), q.stride(0),
                        q.stride(1), out.data_ptr(), out.stride(0), out.stride(1),
                        None if lse is None else lse.data_ptr())
    _check(_launch(cache.device, L.loopspec_window_attention, c, cache._scales_ref, ref, ctypes.byref(a), window, sinks,
                   None if ws is None else ws.data_ptr(), nbytes), "loopspec_window_attention")
    return (out, lse) if return_lse else out


def fork_pages(seq_len, table, parent, refs, caches, prefix_len: int = 0, window: int = 0, sinks: int = 0, room: int = 0):
    """A batch whose row i continues row parent[i] (int32 [children]; outside the rows: none) of the batch seq_len
    [rows], table [rows, pages] over the caches of all layers (PagedCache or QuantizedCache, of equal n_pages and
    page_size).  refs [n_pages]: how many entries name a page (a prefix's pages have theirs from the caller).  A row's
    first child takes its pages over, others share the full ones and get a copy of what the last one holds; pages
    without a child, or that the next position does not see (window, sinks), are let go; every child then holds pages
    for `room` more positions.  What a child appends to it shares with nobody, as far as refs tells: a row that was
    shortened into a page it shares must be forked at that length before it is appended to (its first child, too, then
    gets a copy of that page's rest, and other pages behind it).  table's entries without a page lie outside the cache
    (-1), also those behind a row's last page.  Returns (seq_len, table, refs, short), new int32 tensors: short [1]
    counts the pages that were not to be had, whose entries are -1."""
    caches = list(caches)
    _need(bool(caches), "caches: one or more")
    dev, n_pages, page_size = caches[0].device, caches[0].n_pages, caches[0].page_size
    for c in caches:
        if c.n_pages != n_pages or c.page_size != page_size or c.device != dev:
            raise ValueError("caches: on one device, of equal n_pages and page_size")
    cs, sc = (kind.from_buffer_copy(b"".join([c._raw[i] for c in caches]))
              for i, kind in enumerate((B.PagedCacheC * len(caches), B.PageScalesC * len(caches))))
    n, m = _size(seq_len.shape[0], "seq_len"), _size(parent.shape[0], "parent")
    lens, rows = _ints(seq_len, (n,), dev, "seq_len"), _ints(table, (n, None), dev, "table")
    width = _size(table.shape[1], "table")
    of, counts = _ints(parent, (m,), dev, "parent"), _ints(refs, (n_pages,), dev, "refs")
    prefix_len, window = min(_whole(prefix_len, "prefix_len"), 1 << 30), min(_whole(window, "window"), 1 << 30)
    sinks, room = min(_whole(sinks, "sinks"), 1 << 30), min(_whole(room, "room"), 1 << 30)
    new_len, new_table, new_refs, short = (refs.new_empty(shape) for shape in ((m,), (m, width), (n_pages,), (1,)))
    a = B.ForkArgs(n, m, page_size, n_pages, lens, rows, table.stride(0), width, of, counts, prefix_len, window, sinks, room,
                   new_len.data_ptr(), new_table.data_ptr(), width, new_refs.data_ptr(), short.data_ptr())
    L = B.load_library()
    nbytes = L.loopspec_fork_pages_workspace_bytes(m, n_pages)
    ws = refs.new_empty((nbytes // 4,))         # (whole words)
    _check(_launch(dev, L.loopspec_fork_pages, ctypes.byref(a), cs, sc, len(caches), ws.data_ptr(), nbytes),
           "loopspec_fork_pages")
    return new_len, new_table, new_refs, short


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One token per row of logits [rows, vocab] (float32, bfloat16 or float16; rows may be strided or expanded) with
    the row's uniform number u [rows] (float64, in [0, 1)): temperature (0: the largest logit), then top_k (<= 0:
    all), top_p and min_p (relative to the likeliest token), each a number or a tensor [rows] (float32; top_k int32).
    Returns (tokens int32, their probabilities among the kept ids float32, number of kept ids int32), [rows] each;
    a row that cannot be drawn from (NaN or +infinity, no finite logit, settings out of range) gives (-1, 0, 0)."""
    import torch
    _need(logits.dim() == 2 and logits.is_cuda and _dtype(logits) >= 0, "logits: [rows, vocab] float32, bfloat16 or "
          "float16 on a GPU")
    rows, vocab = (_size(n, "logits") for n in logits.shape)
    dev = logits.device
    _need(vocab == 1 or logits.stride(1) == 1, "logits: a row's elements next to each other")
    _need(u.dtype == torch.float64 and u.shape == (rows,) and u.is_contiguous() and u.device == dev,
          "u: float64 [rows] on the logits' device")
    values, arrays = [], []
    for name, x, kind in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                          ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32)):
        if torch.is_tensor(x):
            _need(x.dtype == kind and x.shape == (rows,) and x.is_contiguous() and x.device == dev,
                  f"{name}: a number or {kind} [rows] on the logits' device")
            values.append(0)
            arrays.append(x.data_ptr())
        else:
            # (more ranks than there are keep all; the field has 32 bits)
            values.append(min(max(operator.index(x), 0), vocab) if kind is torch.int32 else x)
            arrays.append(None)
    cfg = B.SampleCfg(vocab, _dtype(logits), *values, *arrays)
    token = torch.empty((rows,), dtype=torch.int32, device=dev)
    kept, prob = torch.empty_like(token), torch.empty_like(token, dtype=torch.float32)
    L = B.load_library()
    nbytes = L.loopspec_sample_workspace_bytes(vocab, rows)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _check(_launch(dev, L.loopspec_sample, ctypes.byref(cfg), rows, logits.data_ptr(), logits.stride(0), u.data_ptr(),
                   token.data_ptr(), prob.data_ptr(), kept.data_ptr(), ws.data_ptr(), nbytes), "loopspec_sample")
    return token, prob, kept
