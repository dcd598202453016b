"""Serving over a paged K/V cache (include/sra.h, sra_tree_attention and sra_cache_append): argument marshalling.

    o, lse = tree_attention(q, k, v, k_cache, v_cache, page_table, context_lens, cu_tokens, tree)   # every layer
    cache_append(k, v, k_cache, v_cache, page_table, context_lens, cu_tokens_accepted, rows=accepted)
    context_lens += accepted_per_sequence
"""
from __future__ import annotations

import ctypes
from typing import Dict, Optional

import numpy as np

from . import sra as _s
from .causal import INT32_MAX, _addr, _call, _no_alias, _rows

_declared = False


class _PagedCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "tokens", "num_kv_heads", "head_dim", "num_pages", "page_size",
                                              "max_pages")] + \
               [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("k_page_stride", "v_page_stride", "k_token_stride", "v_token_stride")] + \
               [("page_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("context_lens", ctypes.c_void_p),
                ("cu_tokens", ctypes.c_void_p)]


def _lib():
    global _declared
    L = _s.lib()
    if not _declared:
        vp, i32, i64, sz, f = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        pc = ctypes.POINTER(_PagedCache)
        for name, args in {
            "sra_tree_workspace_size": [pc, i32, ctypes.POINTER(sz)],
            "sra_tree_attention": [pc, i32] + [vp] * 3 + [i64] * 3 + [vp] * 3 + [f, vp, sz, vp],
            "sra_cache_append": [pc, vp, vp, i64, i64, vp, i32, vp],
            "sra_cache_rows": [pc, vp, i32, vp],
        }.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        _declared = True
    return L


def _ints(t, name, dims, dtype):
    """An integer tensor of so many dims with contiguous entries."""
    if not isinstance(t, _s._tm().Tensor) or t.dtype != dtype or t.dim() != dims:
        raise _s._bad(f"{name} must be a {dims}-dimensional {dtype} tensor")
    if not t.is_contiguous() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise _s._bad(f"{name}: entries must be contiguous")


def _pages(t, name, shape, kv_heads, head_dim):
    """Page and token strides of a cache tensor (0: it has one page)."""
    torch = _s._tm()
    if not isinstance(t, torch.Tensor) or t.dtype != torch.bfloat16 or len(shape) != 4:
        raise _s._bad(f"{name} must be a bfloat16 [pages, page_size, kv_heads, head_dim] tensor")
    pages, size, heads, dim = shape
    if t.shape != shape or heads != kv_heads or dim != head_dim:
        raise _s._bad(f"{name}: shape {tuple(t.shape)}, expected [pages, page_size, {kv_heads}, {head_dim}]")
    page, token, head, one = t.stride()
    row = heads * dim
    if pages and size:
        if one != 1 or (head != dim and heads > 1):
            raise _s._bad(f"{name} must have contiguous heads")
        if token < row or (pages > 1 and page < (size - 1) * token + row):
            raise _s._bad(f"{name}: tokens or pages overlap")
    return page if pages > 1 else 0, token


def _cache(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens, kv_heads, head_dim):
    """The checked sra_paged_cache of the tensors."""
    torch = _s._tm()
    if not isinstance(k_cache, torch.Tensor):
        raise _s._bad("k_cache must be a torch tensor")
    shape = k_cache.shape
    kp, kt = _pages(k_cache, "k_cache", shape, kv_heads, head_dim)
    vp, vt = _pages(v_cache, "v_cache", shape, kv_heads, head_dim)
    _ints(page_table, "page_table", 2, torch.int32)
    _ints(context_lens, "context_lens", 1, torch.int32)
    _ints(cu_tokens, "cu_tokens", 1, torch.int32)
    n = context_lens.shape[0]
    rows, width = page_table.shape
    if rows != n or cu_tokens.shape[0] != n + 1:
        raise _s._bad("page_table needs one row and cu_tokens one entry more than context_lens has")
    if max(n, tokens, width, *shape[:2]) > INT32_MAX:
        raise _s._bad("sequences, tokens, pages, page_size and page_table entries must be below 2^31")
    ts = page_table.stride(0) if n > 1 else 0
    if n > 1 and ts < width:
        raise _s._bad("page_table: rows overlap")
    return _PagedCache(n, tokens, kv_heads, head_dim, shape[0], shape[1], width, _addr(k_cache), _addr(v_cache),
                       kp, vp, kt, vt, _addr(page_table), ts, _addr(context_lens), _addr(cu_tokens))


def _rows_apart(c, row):
    """Whether no K row of the cache shares memory with a V row (both are written at once): the tensors lie apart, or have
    the same strides and the V rows lie between the K pages, or between their tokens."""
    def end(page, token):
        return 2 * ((c.num_pages - 1) * page + (c.page_size - 1) * token + row)
    d = (c.v or 0) - (c.k or 0)
    if d >= end(c.k_page_stride, c.k_token_stride) or -d >= end(c.v_page_stride, c.v_token_stride):
        return True
    page, token = c.k_page_stride, c.k_token_stride
    if (c.v_token_stride, c.num_pages > 1 and c.v_page_stride) != (token, c.num_pages > 1 and page) or d % 2:
        return False
    d //= 2
    span = (c.page_size - 1) * token + row
    if c.num_pages > 1 and span <= d % page <= page - span:
        return True
    return (c.num_pages == 1 or page % token == 0) and row <= d % token <= token - row


def _dims(t, name):
    if not isinstance(t, _s._tm().Tensor) or t.dim() != 3:
        raise _s._bad(f"{name} must be a [tokens, heads, head_dim] tensor")
    return t.shape


def tree_attention(q, k, v, k_cache, v_cache, page_table, context_lens, cu_tokens, tree=None,
                   scale: Optional[float] = None, out: Optional[Dict] = None):
    """Attention of every sequence's new tokens over its cached context and each other. Returns (o, lse).

    q: bf16 [tokens, heads, head_dim], k, v: the new tokens' bf16 [tokens, kv_heads, head_dim], packed sequence by
    sequence: cu_tokens int32 [batch + 1] are the packed offsets. k_cache, v_cache: bf16 [pages, page_size, kv_heads,
    head_dim] (page_size a power of two, at least 8; pages and tokens may be strided), page_table int32 [batch,
    max_pages], context_lens int32 [batch] cached positions of each sequence, not counting the new tokens. All on q's
    GPU; the call reads them there when it runs, so it can be captured and replayed with other lengths.
    tree: int64 [tokens], bit j of token i's mask = it sees new token j (< 64) of its sequence, itself included only
    if its own bit is set. None: each token sees the new tokens of its sequence up to itself (a single token, or a chain
    of any length).
    o: bf16 like q, dense; lse fp32 [heads, tokens]. Tokens that are no sequence's (before cu_tokens[0], behind
    cu_tokens[-1]) are padding and keep what `out` held.
    Positions in pages outside the cache are seen by no token. An infinity or NaN in v may reach any token of its
    sequence. scale: None or <= 0 selects 1 / sqrt(head_dim). Prompts without a cached context are faster through
    causal_forward (two to three times) than as chains. `out` may hold o, lse and workspace (uint8).
    """
    torch = _s._tm()
    tokens, heads, d = _dims(q, "q")
    kv = _dims(k, "k")[1]
    shape, kv_shape = (tokens, heads, d), (tokens, kv, d)
    qs, ks, vs = _rows(q, "q", shape), _rows(k, "k", kv_shape), _rows(v, "v", kv_shape)
    c = _cache(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens, kv, d)
    if tree is not None:
        _ints(tree, "tree", 1, torch.int64)
        if tree.shape[0] != tokens:
            raise _s._bad("tree needs one mask per token")
    if out:
        _s._precheck_outs(out, [("o", shape, torch.bfloat16), ("lse", (heads, tokens), torch.float32)])
    nbytes = _workspace_size(c, heads)
    dev = q.device
    ins = (("q", q), ("k", k), ("v", v), ("tree", tree), ("k_cache", k_cache), ("v_cache", v_cache),
           ("page_table", page_table), ("context_lens", context_lens), ("cu_tokens", cu_tokens))
    _s._same_device(ins, dev)
    if out:
        o = _s._out(out, "o", shape, torch.bfloat16, dev)
        lse = _s._out(out, "lse", (heads, tokens), torch.float32, dev)
        ws = _s._workspace(out, nbytes, dev)
        _no_alias(out, ins + (("o", o), ("lse", lse), ("workspace", ws)))
    else:
        o = torch.empty(shape, dtype=torch.bfloat16, device=dev)
        lse = torch.empty((heads, tokens), dtype=torch.float32, device=dev)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _s._check(_call(dev, lambda s: _lib().sra_tree_attention(
        c, heads, _addr(q), _addr(k), _addr(v), qs, ks, vs, _addr(tree), _addr(o), _addr(lse),
        0.0 if scale is None else float(scale), ws.data_ptr(), ws.numel(), s)))
    return o, lse


_SIZES: Dict[tuple, int] = {}


def _workspace_size(c, heads):
    """sra_tree_workspace_size, asked once per set of sizes."""
    key = (c.batch, c.tokens, c.num_kv_heads, c.head_dim, c.num_pages, c.page_size, c.max_pages, c.table_stride,
           c.k_page_stride, c.v_page_stride, c.k_token_stride, c.v_token_stride, heads)
    n = _SIZES.get(key)
    if n is None:
        size = ctypes.c_size_t()
        _s._check(_lib().sra_tree_workspace_size(c, heads, ctypes.byref(size)))
        if len(_SIZES) >= 4096:
            _SIZES.clear()
        n = _SIZES[key] = size.value
    return n


def cache_append(k, v, k_cache, v_cache, page_table, context_lens, cu_tokens, rows=None):
    """Writes K and V of new tokens into the cache, behind their sequences' context: token i of sequence b goes to
    position context_lens[b] + i - cu_tokens[b]. The cache is changed in place; context_lens is the caller's to advance.

    k, v: bf16 [n, kv_heads, head_dim]; without `rows` their rows are the packed tokens. rows: int32 [tokens], the row
    of k and v that each packed token is (the accepted tokens of a drafted tree). Cache, page_table, context_lens and
    cu_tokens as for tree_attention; k_cache and v_cache must not share rows. Tokens behind the page_table row, in a page
    outside the cache or with a row outside k and v are skipped.
    """
    n, kv, d = _dims(k, "k")
    ks, vs = _rows(k, "k", (n, kv, d)), _rows(v, "v", (n, kv, d))
    tokens = n
    if rows is not None:
        _ints(rows, "rows", 1, _s._tm().int32)
        tokens = rows.shape[0]
    c = _cache(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens, kv, d)
    dev = k.device
    if not _rows_apart(c, kv * d):
        raise _s._bad("k_cache and v_cache overlap")
    if n and c.num_pages:  # rows are read while others are written
        spans = [(t.data_ptr(), t.data_ptr() + 2 * ((t.shape[0] - 1) * s + kv * d)) for t, s in ((k, ks), (v, vs))]
        for cache, ps, ts in ((k_cache, c.k_page_stride, c.k_token_stride), (v_cache, c.v_page_stride, c.v_token_stride)):
            a = cache.data_ptr()
            b = a + 2 * ((c.num_pages - 1) * ps + (c.page_size - 1) * ts + kv * d)
            if any(lo < b and a < hi for lo, hi in spans):
                raise _s._bad("k or v overlaps the cache")
    _s._same_device((("k", k), ("v", v), ("rows", rows), ("k_cache", k_cache), ("v_cache", v_cache),
                     ("page_table", page_table), ("context_lens", context_lens), ("cu_tokens", cu_tokens)), dev)
    _s._check(_call(dev, lambda s: _lib().sra_cache_append(c, _addr(k), _addr(v), ks, vs, _addr(rows), n, s)))


def cache_rows(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens: int, sequence: int = 0):
    """sra_cache_rows on CPU tensors: (the cache row that each of `tokens` packed tokens is appended to, the cache rows
    of the positions of `sequence` up to its page_table row's end), -1 where there is none."""
    kv, d = _cache_dims(k_cache)
    c = _cache(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens, kv, d)
    for name, t in (("page_table", page_table), ("context_lens", context_lens), ("cu_tokens", cu_tokens)):
        if t.device.type != "cpu":
            raise _s._bad(f"{name}: the hook reads host memory")
    a = np.full(max(tokens, 1), -1, dtype=np.int64)
    p = np.full(max(page_table.shape[1] * k_cache.shape[1], 1), -1, dtype=np.int64)
    _s._check(_lib().sra_cache_rows(c, a.ctypes.data, sequence, p.ctypes.data))
    return a[:tokens], p


def _cache_dims(k_cache):
    if not isinstance(k_cache, _s._tm().Tensor) or k_cache.dim() != 4:
        raise _s._bad("k_cache must be a [pages, page_size, kv_heads, head_dim] tensor")
    return k_cache.shape[2:]
