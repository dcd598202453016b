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
from .causal import _call, _no_alias, _stride

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


def _ints(t, name, dims):
    """An int32 tensor of so many dims (or, 8 bytes wide, the tree masks) with contiguous entries."""
    torch = _s._tm()
    want = torch.int64 if name == "tree" else torch.int32
    if not isinstance(t, torch.Tensor) or t.dtype != want or t.dim() != dims:
        raise _s._bad(f"{name} must be a {dims}-dimensional {want} tensor")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise _s._bad(f"{name}: entries must be contiguous")


def _cache(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens, kv_heads, head_dim):
    """The checked sra_paged_cache of the tensors."""
    torch = _s._tm()
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        if not isinstance(t, torch.Tensor) or t.dtype != torch.bfloat16 or t.dim() != 4:
            raise _s._bad(f"{name} must be a bfloat16 [pages, page_size, kv_heads, head_dim] tensor")
        if t.shape != k_cache.shape or t.shape[2:] != (kv_heads, head_dim):
            raise _s._bad(f"{name}: shape {tuple(t.shape)}, expected [pages, page_size, {kv_heads}, {head_dim}]")
        if t.numel() and (t.stride(3) != 1 or (kv_heads > 1 and t.stride(2) != head_dim)):
            raise _s._bad(f"{name} must have contiguous heads")
        if t.numel() and (t.stride(1) < kv_heads * head_dim or
                          (t.shape[0] > 1 and t.stride(0) < (t.shape[1] - 1) * t.stride(1) + kv_heads * head_dim)):
            raise _s._bad(f"{name}: tokens or pages overlap")
    _ints(page_table, "page_table", 2)
    _ints(context_lens, "context_lens", 1)
    _ints(cu_tokens, "cu_tokens", 1)
    n = context_lens.shape[0]
    if page_table.shape[0] != n or cu_tokens.shape[0] != n + 1:
        raise _s._bad("page_table needs one row and cu_tokens one entry more than context_lens has")
    if n > 1 and page_table.stride(0) < page_table.shape[1]:
        raise _s._bad("page_table: rows overlap")
    pages, page = k_cache.shape[:2]
    # a single page (or token of a page) has no stride of its own
    kp, vp = (t.stride(0) if pages > 1 else 0 for t in (k_cache, v_cache))
    c = _PagedCache(n, tokens, kv_heads, head_dim, pages, page, page_table.shape[1], _addr(k_cache), _addr(v_cache),
                    kp, vp, k_cache.stride(1), v_cache.stride(1), _addr(page_table),
                    page_table.stride(0) if n > 1 else 0, _addr(context_lens), _addr(cu_tokens))
    return c, (("k_cache", k_cache), ("v_cache", v_cache), ("page_table", page_table), ("context_lens", context_lens),
               ("cu_tokens", cu_tokens))


def _addr(t):
    return t.data_ptr() if t is not None and t.numel() else None


def _end(t):
    return t.data_ptr() + t.element_size() * (sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1)


def _rows(t, name, shape):
    _s._expect(t, name, shape, _s._tm().bfloat16, False)
    return _stride(t, name)


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
    o: bf16 like q, dense; lse fp32 [heads, tokens]. Tokens behind cu_tokens[-1] are padding and keep what `out` held.
    Positions in pages outside the cache are seen by no token. `out` may hold o, lse and workspace (uint8).
    """
    torch = _s._tm()
    tokens, heads, d = _dims(q, "q")
    kv = _dims(k, "k")[1]
    qs, ks, vs = _rows(q, "q", (tokens, heads, d)), _rows(k, "k", (tokens, kv, d)), _rows(v, "v", (tokens, kv, d))
    c, tensors = _cache(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens, kv, d)
    if tree is not None:
        _ints(tree, "tree", 1)
        if tree.shape[0] != tokens:
            raise _s._bad("tree needs one mask per token")
    _s._precheck_outs(out, [("o", (tokens, heads, d), torch.bfloat16), ("lse", (heads, tokens), torch.float32)])
    n = ctypes.c_size_t()
    _s._check(_lib().sra_tree_workspace_size(ctypes.byref(c), heads, ctypes.byref(n)))
    dev = q.device
    ins = (("q", q), ("k", k), ("v", v), ("tree", tree)) + tensors
    _s._same_device(ins, dev)
    out = out or {}
    o = _s._out(out, "o", (tokens, heads, d), torch.bfloat16, dev)
    lse = _s._out(out, "lse", (heads, tokens), torch.float32, dev)
    ws = _s._workspace(out, n.value, dev)
    if out:
        _no_alias(out, ins + (("o", o), ("lse", lse), ("workspace", ws)))
    _s._check(_call(dev, lambda s: _lib().sra_tree_attention(
        ctypes.byref(c), heads, _addr(q), _addr(k), _addr(v), qs, ks, vs, _addr(tree), _addr(o), _addr(lse),
        0.0 if scale is None else float(scale), _addr(ws), ws.numel(), s)))
    return o, lse


def cache_append(k, v, k_cache, v_cache, page_table, context_lens, cu_tokens, rows=None):
    """Writes K and V of new tokens into the cache, behind their sequences' context: token i of sequence b goes to
    position context_lens[b] + i - cu_tokens[b]. The cache is changed in place; context_lens is the caller's to advance.

    k, v: bf16 [n, kv_heads, head_dim]; without `rows` their rows are the packed tokens. rows: int32 [tokens], the row
    of k and v that each packed token is (the accepted tokens of a drafted tree). Cache, page_table, context_lens and
    cu_tokens as for tree_attention. Tokens behind the page_table row, in a page outside the cache or with a row outside
    k and v are skipped.
    """
    n, kv, d = _dims(k, "k")
    ks, vs = _rows(k, "k", (n, kv, d)), _rows(v, "v", (n, kv, d))
    tokens = n
    if rows is not None:
        _ints(rows, "rows", 1)
        tokens = rows.shape[0]
    c, tensors = _cache(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens, kv, d)
    dev = k.device
    ins = (("k", k), ("v", v), ("rows", rows)) + tensors
    for name, t in (("k", k), ("v", v)):  # rows are read while others are written
        for other, cache in tensors[:2]:
            if t.numel() and cache.numel() and _end(t) > cache.data_ptr() and _end(cache) > t.data_ptr():
                raise _s._bad(f"{name} overlaps {other}")
    _s._same_device(ins, dev)
    _s._check(_call(dev, lambda s: _lib().sra_cache_append(ctypes.byref(c), _addr(k), _addr(v), ks, vs, _addr(rows), n, s)))


def cache_rows(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens: int, sequence: int = 0):
    """sra_cache_rows on CPU tensors: (the cache row that each of `tokens` packed tokens is appended to, the cache rows
    of the positions of `sequence` up to its page_table row's end), -1 where there is none."""
    kv, d = _cache_dims(k_cache)
    c, tensors = _cache(k_cache, v_cache, page_table, context_lens, cu_tokens, tokens, kv, d)
    for name, t in tensors[2:]:
        if t.device.type != "cpu":
            raise _s._bad(f"{name}: the hook reads host memory")
    a = np.full(max(tokens, 1), -1, dtype=np.int64)
    p = np.full(max(page_table.shape[1] * k_cache.shape[1], 1), -1, dtype=np.int64)
    _s._check(_lib().sra_cache_rows(ctypes.byref(c), a.ctypes.data, sequence, p.ctypes.data))
    return a[:tokens], p


def _cache_dims(k_cache):
    if not isinstance(k_cache, _s._tm().Tensor) or k_cache.dim() != 4:
        raise _s._bad("k_cache must be a [pages, page_size, kv_heads, head_dim] tensor")
    return k_cache.shape[2:]
