"""The paged cache on the host: where tokens and positions lie, also for bad pages and lengths, and every refusal."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_13872_amd as sra
from oracle import text_oracle as T
from paper_2606_13872_amd import cache as binding

I32 = torch.int32


def cache(pages=6, page=8, kv=2, d=64):
    return torch.zeros(pages, page, kv, d, dtype=torch.bfloat16)


def rows(table, ctx, cu, tokens, sequence=0, pages=6, page=8):
    c = cache(pages, page)
    return sra.cache_rows(c, c, torch.tensor(table, dtype=I32), torch.tensor(ctx, dtype=I32), torch.tensor(cu, dtype=I32),
                          tokens, sequence)


def test_tokens_and_positions_lie_where_the_table_says():
    a, p = rows([[3, 0], [5, 2]], [6, 0], [0, 4, 7], 9, sequence=0)
    assert a.tolist() == [3 * 8 + 6, 3 * 8 + 7, 0, 1, 5 * 8, 5 * 8 + 1, 5 * 8 + 2, -1, -1]  # the last two: padding
    assert p.tolist() == [24 + i for i in range(6)] + [-1] * 10


def test_bad_pages_and_lengths_have_no_place():
    a, p = rows([[3, -1], [6, 2]], [7, 14], [0, 3, 6], 6)
    assert a.tolist() == [31, -1, -1, 22, 23, -1]        # page -1; then the end of the second table row
    assert rows([[3, -1], [6, 2]], [16, 9], [0, 3, 6], 6, 0)[1].tolist() == [24 + i for i in range(8)] + [-1] * 8
    assert rows([[3, -1], [6, 2]], [16, 9], [0, 3, 6], 6, 1)[1].tolist() == [-1] * 8 + [16] + [-1] * 7
    big = 2**31 - 1
    assert rows([[1, 2]], [big], [0, 3], 3)[0].tolist() == [-1] * 3
    assert rows([[1, 2]], [big], [0, 3], 3)[1].tolist() == [8 + i for i in range(16)]  # the table row's reach
    assert rows([[1, 2]], [-4], [0, 3], 3)[0].tolist() == [8, 9, 10]
    assert rows([[1, 2]], [-4], [0, 3], 3)[1].tolist() == [-1] * 16
    # offsets outside the packed tokens, and falling ones
    assert rows([[1, 2]], [0], [-2, 100], 3)[0].tolist() == [8, 9, 10]
    assert (rows([[1, 2], [3, 4]], [0, 0], [2, 1, 3], 3)[0][:1] == -1).all()


def test_definition_reads_the_cache_it_is_given():
    """The float64 definition: a tree over a paged context equals causal attention of the same tokens laid out plainly."""
    g = torch.Generator().manual_seed(0)
    kv, d, page, ctx = 2, 16, 8, 21
    k, v = (torch.randn(ctx + 3, kv, d, generator=g, dtype=torch.float64) for _ in range(2))
    q = torch.randn(3, 4, d, generator=g, dtype=torch.float64)
    table = torch.tensor([[4, 1, 2]], dtype=I32)
    kc, vc = (torch.full((6, page, kv, d), float("nan"), dtype=torch.float64) for _ in range(2))
    pos = torch.arange(ctx)
    kc[table[0].long()[pos // page], pos % page], vc[table[0].long()[pos // page], pos % page] = k[:ctx], v[:ctx]
    val, _ = T.tree(q, k[ctx:], v[ctx:], kc, vc, table, [ctx], [0, 3], [1, 3, 7])
    chain, _ = T.tree(q, k[ctx:], v[ctx:], kc, vc, table, [ctx], [0, 3])
    want, _ = T.causal(q, k, v, [3], [ctx + 3])
    for x in (val, chain):
        assert float((x["o"] - want["o"]).abs().max()) < 1e-12 and float((x["lse"] - want["lse"]).abs().max()) < 1e-12
    wrong, _ = T.tree(q, k[ctx:], v[ctx:], kc, vc, table, [ctx], [0, 3], [1, 3, 3])  # a planted mask mistake
    assert float((wrong["o"][2] - want["o"][2]).abs().max()) > 1e-3


def step(tokens=5, heads=4, kv=2, d=64, batch=2):
    bf = torch.bfloat16
    return dict(q=torch.zeros(tokens, heads, d, dtype=bf), k=torch.zeros(tokens, kv, d, dtype=bf),
                v=torch.zeros(tokens, kv, d, dtype=bf), k_cache=cache(kv=kv, d=d), v_cache=cache(kv=kv, d=d),
                page_table=torch.zeros(batch, 3, dtype=I32), context_lens=torch.zeros(batch, dtype=I32),
                cu_tokens=torch.zeros(batch + 1, dtype=I32))


BAD = {
    "q dtype": dict(q=torch.zeros(5, 4, 64)),
    "q rank": dict(q=torch.zeros(5, 256, dtype=torch.bfloat16)),
    "k tokens": dict(k=torch.zeros(4, 2, 64, dtype=torch.bfloat16)),
    "v heads": dict(v=torch.zeros(5, 4, 64, dtype=torch.bfloat16)),
    "heads not a multiple": dict(q=torch.zeros(5, 3, 64, dtype=torch.bfloat16)),
    "cache dtype": dict(k_cache=torch.zeros(6, 8, 2, 64)),
    "cache shapes differ": dict(v_cache=cache(pages=7)),
    "cache heads": dict(k_cache=cache(kv=3), v_cache=cache(kv=3)),
    "cache head layout": dict(k_cache=torch.zeros(6, 2, 8, 64, dtype=torch.bfloat16).transpose(1, 2)),
    "overlapping pages": dict(k_cache=cache(pages=1).expand(6, 8, 2, 64)),
    "page size 12": dict(k_cache=cache(page=12), v_cache=cache(page=12)),
    "page size 4": dict(k_cache=cache(page=4), v_cache=cache(page=4)),
    "no pages": dict(k_cache=cache(pages=0), v_cache=cache(pages=0)),
    "table dtype": dict(page_table=torch.zeros(2, 3, dtype=torch.int64)),
    "table rank": dict(page_table=torch.zeros(6, dtype=I32)),
    "table columns": dict(page_table=torch.zeros(3, 2, dtype=I32).t()),
    "table rows": dict(page_table=torch.zeros(3, 3, dtype=I32)),
    "empty table": dict(page_table=torch.zeros(2, 0, dtype=I32)),
    "lens dtype": dict(context_lens=torch.zeros(2, dtype=torch.int64)),
    "cu length": dict(cu_tokens=torch.zeros(2, dtype=I32)),
    "tree dtype": dict(tree=torch.zeros(5, dtype=I32)),
    "tree length": dict(tree=torch.zeros(4, dtype=torch.int64)),
    "no sequences": dict(page_table=torch.zeros(0, 3, dtype=I32), context_lens=torch.zeros(0, dtype=I32),
                         cu_tokens=torch.zeros(1, dtype=I32)),
    "out dtype": dict(out={"o": torch.zeros(5, 4, 64)}),
    "out shape": dict(out={"lse": torch.zeros(5, 4)}),
    "scale": dict(scale=float("nan")),
    "cpu tensors": dict(),
}


@pytest.mark.parametrize("name", list(BAD))
def test_bad_steps_are_refused(name):
    with pytest.raises(sra.SRAError) as e:
        sra.tree_attention(**{**step(), **BAD[name]})
    assert e.value.status == 1


def test_sizes_the_library_does_not_serve():
    with pytest.raises(sra.SRAError) as e:
        sra.tree_attention(**step(batch=2049))
    assert e.value.status == 2
    with pytest.raises(sra.SRAError) as e:
        sra.tree_attention(**step(d=96))
    assert e.value.status == 2


def test_bad_appends_are_refused():
    s = step()
    args = [s[n] for n in ("k", "v", "k_cache", "v_cache", "page_table", "context_lens", "cu_tokens")]

    def bad(status=1, rows=None, **kw):
        names = ("k", "v", "k_cache", "v_cache", "page_table", "context_lens", "cu_tokens")
        with pytest.raises(sra.SRAError) as e:
            sra.cache_append(*(kw.get(n, a) for n, a in zip(names, args)), rows=rows)
        assert e.value.status == status

    bad()  # on the CPU
    bad(v=torch.zeros(4, 2, 64, dtype=torch.bfloat16))
    bad(k=torch.zeros(5, 2, 64))
    bad(rows=torch.zeros(5, dtype=torch.int64))
    bad(rows=torch.zeros(5, 1, dtype=I32))
    bad(cu_tokens=torch.zeros(2, dtype=I32))
    bad(k=args[2].view(-1, 2, 64)[:5])  # rows of the cache itself
    bad(k_cache=cache(d=128))


def test_library_refuses_before_any_launch():
    L = binding._lib()
    fake, null, odd = 1 << 20, None, (1 << 20) + 2

    def paged(**kw):
        f = dict(batch=2, tokens=5, num_kv_heads=2, head_dim=64, num_pages=6, page_size=8, max_pages=3, k=fake, v=fake,
                 k_page_stride=0, v_page_stride=0, k_token_stride=0, v_token_stride=0, page_table=fake, table_stride=0,
                 context_lens=fake, cu_tokens=fake)
        f.update(kw)
        return binding._PagedCache(*(f[n] for n, _ in binding._PagedCache._fields_))

    def tree(heads=4, q=fake, k=fake, o=fake, qs=0, ks=0, mask=null, scale=0.0, ws=fake, n=1 << 30, **kw):
        return L.sra_tree_attention(ctypes.byref(paged(**kw)), heads, q, k, fake, qs, ks, 0, mask, o, fake, scale, ws, n, null)

    def append(k=fake, ks=0, rows=null, n=5, **kw):
        return L.sra_cache_append(ctypes.byref(paged(**kw)), k, fake, ks, 0, rows, n, null)

    for call in (tree, append):
        for kw in (dict(batch=0), dict(tokens=-1), dict(num_kv_heads=0), dict(head_dim=0), dict(num_pages=0), dict(page_size=12),
                   dict(page_size=4), dict(page_size=0), dict(max_pages=0), dict(k=null) if call is tree else dict(v=null),
                   dict(k_page_stride=8 * 128 - 8), dict(v_page_stride=8 * 128 + 4), dict(k_token_stride=64),
                   dict(v_token_stride=132), dict(page_table=null), dict(page_table=odd), dict(table_stride=2),
                   dict(context_lens=null), dict(cu_tokens=odd)):
            assert call(**kw) == 1, (call, kw)
        for kw in (dict(batch=2049), dict(head_dim=96), dict(k_token_stride=1 << 34), dict(v_page_stride=1 << 50),
                   dict(max_pages=1 << 28), dict(tokens=2**31 - 1)):
            assert call(**kw) == 2, (call, kw)
    assert tree(heads=3) == 1 and tree(q=null) == 1 and tree(k=odd) == 1 and tree(o=null) == 1 and tree(mask=odd) == 1
    assert tree(qs=128) == 1 and tree(ks=68) == 1 and tree(scale=float("inf")) == 1 and tree(ws=odd) == 1 and tree(n=16) == 3
    # 2^31 chunks and more in one launch
    assert tree(tokens=2**20, max_pages=2**27) == 2
    assert append(k=null) == 1 and append(n=4) == 1 and append(rows=odd) == 1 and append(ks=64) == 1 and append(rows=fake, n=-1) == 1
    assert tree(tokens=0) == 0 and append(tokens=0, n=0) == 0  # nothing to do, nothing launched
    assert L.sra_cache_rows(ctypes.byref(paged()), null, 2, fake) == 1
    n = ctypes.c_size_t()
    assert L.sra_tree_workspace_size(ctypes.byref(paged(k=null, page_table=null)), 4, ctypes.byref(n)) == 0 and n.value % 256 == 0
    assert L.sra_tree_workspace_size(ctypes.byref(paged()), 4, null) == 1


@pytest.mark.parametrize("apart,layout", [
    (True, lambda x: (x[0, :, 0], x[1, :, 0])),              # two buffers
    (True, lambda x: (x[0, :, 0], x[0, :, 1])),              # K and V pages in turn
    (True, lambda x: (x[0, :, 1], x[0, :, 0])),
    (True, lambda x: (x[0].view(4, 16, 2, 2, 64)[:, :, 0], x[0].view(4, 16, 2, 2, 64)[:, :, 1])),  # tokens in turn
    (True, lambda x: (x[0, :1, 0], x[0, :1, 1])),            # one page
    (False, lambda x: (x[0, :, 0], x[0, :, 0])),             # the same one
    (False, lambda x: (x[0].flatten(0, 1)[:4], x[0].flatten(0, 1)[1:5])),  # a page further
    (False, lambda x: (x[0, :, 0], x[0].flatten(0, 1)[1:5])),  # other strides
    (False, lambda x: (x[0, :1, 0], x.view(-1)[128:128 + 2048].view(1, 16, 2, 64))),  # a token further
])
def test_an_append_needs_its_own_rows_for_keys_and_values(apart, layout):
    k, v = layout(torch.zeros(2, 4, 2, 16, 2, 64, dtype=torch.bfloat16))
    new = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    c = binding._cache(k, v, torch.tensor([[0]], dtype=I32), torch.tensor([1], dtype=I32), torch.tensor([0, 3], dtype=I32),
                       3, 2, 64)
    assert binding._rows_apart(c, 128) == apart
    if not apart:
        with pytest.raises(sra.SRAError, match="overlap"):
            sra.cache_append(new, new.clone(), k, v, torch.tensor([[0]], dtype=I32), torch.tensor([1], dtype=I32),
                             torch.tensor([0, 3], dtype=I32))


def test_more_tokens_than_a_launch_takes_are_refused():
    k = torch.zeros(1, 1, 64, dtype=torch.bfloat16).expand(2**25 + 1, 1, 64)
    c = cache(kv=1)
    args = (torch.tensor([[0]], dtype=I32), torch.tensor([1], dtype=I32), torch.tensor([0, 3], dtype=I32))
    paged = binding._cache(c, c, *args, k.shape[0], 1, 64)
    with pytest.raises(sra.SRAError) as e:
        binding._workspace_size(paged, 1)
    assert e.value.status == 2
