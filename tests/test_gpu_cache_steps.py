"""Steps over a paged cache that mix what a server mixes, on the GPU against the float64 definitions (oracle/text_oracle.py):
chains of thousands of tokens, long sequences among single tokens, lengths outside their range, infinite and NaN neighbours."""
import math

import pytest
import torch

import paper_2606_13872_amd as sra
from oracle import text_oracle as T
from test_gpu_cache import check, make

pytestmark = pytest.mark.gpu


def _check_chains(x, o, lse, ctx, cu, heads):
    """A chain is the end of a causal sequence: each sequence's rows for some heads."""
    kv, d = x["k"].shape[1:]
    for b, c in enumerate(ctx):
        at = slice(cu[b], cu[b + 1])
        t = cu[b + 1] - cu[b]
        if t == 0:
            continue
        kc, vc = (T.gather_cache(x[n], x["page_table"][b], c) for n in ("k_cache", "v_cache"))
        see = T.causal_mask(t, c + t, "cuda")
        for h in sorted({0, heads // 2, heads - 1}):
            g = h * kv // heads
            k, v = (torch.cat([a[:, g], x[n][at, g]]).double() for a, n in ((kc, "k"), (vc, "v")))
            want, want_lse, _, eo, el = T.rows(x["q"][at, h].double(), k, v, see, 1 / math.sqrt(d))
            for name, got, w, e in (("o", o[at, h], want, eo), ("lse", lse[h, at], want_lse, el)):
                ok, worst = T.within(got, w, e)
                assert ok, f"{name} of sequence {b}, head {h}: {worst:.2f} bounds off"


@pytest.mark.parametrize("heads,kv,d,page", [(8, 2, 128, 16), (4, 4, 64, 8), (3, 1, 64, 64)])
@pytest.mark.parametrize("ctx,new", [([0], [2100]), ([300, 0, 8000], [4099, 65, 513]), ([31, 64], [1023, 1])])
def test_long_chains(ctx, new, heads, kv, d, page):
    print("long chain", ctx, new, heads, kv, d, page, flush=True)
    x, _, cu = make(ctx, new, heads, kv, d, page, seed=60 + heads)
    o, lse = sra.tree_attention(**x)
    _check_chains(x, o, lse, ctx, cu, heads)


# few rows a sequence on average, 32, and more, each with one sequence far from the average
MIXED = [(128, 256), (63, 200), (64, 512), (300, 70)]


@pytest.mark.parametrize("singles,long", MIXED)
@pytest.mark.parametrize("d", [64, 128])
def test_a_long_chain_among_single_tokens(singles, long, d):
    print("mixed", singles, long, d, flush=True)
    at = singles // 3
    ctx = [(37 * i) % 700 for i in range(singles)]
    new = [1] * singles
    ctx.insert(at, 2100)
    new.insert(at, long)
    x, _, cu = make(ctx, new, 8, 2, d, 16, seed=70 + singles)
    o, lse = sra.tree_attention(**x)
    _check_chains(x, o, lse, ctx, cu, 8)
    again = sra.tree_attention(**x)
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)


@pytest.mark.parametrize("singles,long", [(60, 64), (20, 60)])
def test_a_drafted_tree_among_single_tokens(singles, long):
    print("mixed tree", singles, long, flush=True)
    ctx = [(41 * i) % 500 for i in range(singles)] + [1500]
    x, tree, cu = make(ctx, [1] * singles + [long], 8, 2, 128, 16, seed=80)
    check(x, tree, ctx, cu)


def test_lengths_outside_their_range_are_taken_as_the_nearest_ones():
    print("clamped lengths", flush=True)
    x, tree, _ = make([64, 64, 64], [2, 2, 2], 4, 2, 64, 16, seed=8, width=4)

    def same(masks, ctx, cu, heads=4):
        """The call against the definition of these lengths."""
        out = {"o": torch.full_like(x["q"], 5.0), "lse": torch.full((heads, 6), 5.0, device="cuda")}
        sra.tree_attention(**x, tree=masks, out=out)
        bits = None if masks is None else masks.tolist()
        val, bound = T.tree(x["q"], x["k"], x["v"], x["k_cache"], x["v_cache"], x["page_table"], ctx, cu, bits)
        mine = ~torch.isnan(val["lse"][0])
        for n, got, w, e in (("o", out["o"][mine], val["o"][mine], bound["o"][mine]),
                             ("lse", out["lse"][:, mine], val["lse"][:, mine], bound["lse"][:, mine])):
            ok, worst = T.within(got, w, e)
            assert ok, f"{n}: {worst:.2f} bounds off"
        assert bool((out["o"][~mine] == 5).all()) and bool((out["lse"][:, ~mine] == 5).all())

    masks = torch.tensor([1, 3, 1, 3, 5, 15], device="cuda")
    for m in (masks, None):
        x["cu_tokens"][:] = torch.tensor([0, 2, 4, 6])
        x["context_lens"][:] = torch.tensor([64, -5, 10**9])
        same(m, [64, 0, 64], [0, 2, 4, 6])
        x["context_lens"][:] = torch.tensor([-2**31, 64, 2**31 - 1])
        same(m, [0, 64, 64], [0, 2, 4, 6])
        x["context_lens"][:] = 64
        x["cu_tokens"][:] = torch.tensor([-3, 2, 1, 100])  # falling: sequence 1 has nothing, sequence 2 the rest
        same(m, [64, 64, 64], [0, 2, 2, 6])
        x["cu_tokens"][:] = torch.tensor([1, 3, 3, 5])     # padding at both ends, a sequence without tokens
        same(m, [64, 64, 64], [1, 3, 3, 5])
        x["cu_tokens"][:] = torch.tensor([7, 9, 3, 2**31 - 1])
        same(m, [64, 64, 64], [6, 6, 6, 6])                # all of them behind the packed tokens


@pytest.mark.parametrize("new,heads", [([1, 1, 1, 1], 8), ([7, 5, 1, 3], 8), ([40, 64, 33, 31], 8), ([200, 70, 65, 3], 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_infinities_and_nan_stay_in_their_sequence(new, heads, d):
    """Bitwise: rows of other sequences do not change with what a sequence's queries, new tokens and pages hold."""
    print("tree poison", new, heads, d, flush=True)
    ctx = [63, 129, 31, 300]
    x, tree, cu = make(ctx, new, heads, 2, d, 16, seed=90)
    if max(new) > 64:
        tree = None
    o, lse = sra.tree_attention(**x, tree=tree)
    for b in range(4):
        for bad in (math.inf, -math.inf, math.nan):
            y = {n: t.clone() for n, t in x.items()}
            at = slice(cu[b], cu[b + 1])
            for n in ("q", "k", "v"):
                y[n][at] = bad
            pages = y["page_table"][b].long()
            pages = pages[pages >= 0]
            y["k_cache"][pages], y["v_cache"][pages] = bad, bad
            got = sra.tree_attention(**y, tree=tree)
            keep = torch.ones(cu[-1], dtype=torch.bool, device="cuda")
            keep[at] = False
            assert torch.equal(got[0][keep], o[keep]) and torch.equal(got[1][:, keep], lse[:, keep]), (b, bad)


@pytest.mark.parametrize("heads,kv,d,new", [(1024, 1, 64, [1, 2]), (1000, 1, 64, [3]), (77, 7, 128, [1, 13, 2]), (37, 1, 64, [1, 1, 1])])
def test_many_heads_of_one_key_head(heads, kv, d, new):
    """Tokens whose heads take several groups of rows, and groups that begin and end inside a token's heads."""
    print("wide groups", heads, kv, d, new, flush=True)
    ctx = [70, 333, 0][:len(new)]
    x, tree, cu = make(ctx, new, heads, kv, d, 16, seed=100)
    check(x, tree, ctx, cu)


@pytest.mark.parametrize("new", [[1, 1, 1], [9, 30, 20]])
def test_sequences_that_share_pages_and_pages_larger_than_a_context(new):
    print("shared pages", new, flush=True)
    ctx = [200, 640, 513]
    for page in (32, 1024):
        x, tree, cu = make(ctx, new, 8, 2, 128, page, seed=110)
        for n in (1, 2):  # the first positions of all three lie in the first sequence's pages
            x["page_table"][n, :192 // page] = x["page_table"][0, :192 // page]
        check(x, tree, ctx, cu)


def test_new_tokens_as_views_of_one_projection():
    """q, k and v of one buffer give what dense copies give, to the attention and to the append."""
    print("views", flush=True)
    ctx, new = [60, 0, 200], [3, 40, 1]
    for d in (64, 128):
        x, tree, cu = make(ctx, new, 8, 2, d, 16, seed=120)
        buf = torch.cat([x["q"], x["k"], x["v"]], dim=1)
        views = {"q": buf[:, :8], "k": buf[:, 8:10], "v": buf[:, 10:]}
        want = sra.tree_attention(**x, tree=tree)
        got = sra.tree_attention(**{**x, **views}, tree=tree)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        where = [x[n] for n in ("page_table", "context_lens", "cu_tokens")]
        caches = [[x[n].clone() for n in ("k_cache", "v_cache")] for _ in range(2)]
        sra.cache_append(x["k"], x["v"], *caches[0], *where)
        sra.cache_append(views["k"], views["v"], *caches[1], *where)
        for a, b in zip(*caches):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
            assert not torch.equal(a.view(torch.int16), x["k_cache"].view(torch.int16))
