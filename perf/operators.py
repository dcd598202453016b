"""Performance cases of the language-model operators: causal attention over packed prompts, attention
of drafted tokens over a paged cache, and appending to that cache.

A case names its operator ("op") and sizes. "forward" and "step" are causal attention with grouped heads
(inference; training: forward, then the gradients of its outputs), "tree" is the attention of a serving step
(each sequence's new tokens, one or a tree of drafted ones, over its cached context and each other), "append"
writes the K/V of a prompt or of accepted drafts into the cache's pages.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # run() calls the framework's operators (true) or computes their plain form (false)

BLOCK = 1 << 27  # scores of one block of rows in the plain forms: 0.5 GiB in float32


def _causal(name, op, heads, kv_heads, dim, q_lens, k_lens="", packed=False):
    c = {"op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, "q_lens": q_lens, "k_lens": k_lens,
         "packed": packed}
    return c if name is None else {"name": name, **c}


def _tree(name, heads, kv_heads, dim, page, contexts, tokens):
    c = {"op": "tree", "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "contexts": contexts,
         "tokens": tokens}
    return c if name is None else {"name": name, **c}


def _append(name, kv_heads, dim, page, contexts, tokens, picked):
    c = {"op": "append", "kv_heads": kv_heads, "dim": dim, "page": page, "contexts": contexts, "tokens": tokens,
         "picked": picked}
    return c if name is None else {"name": name, **c}


def _text(values):
    return ",".join(map(str, values))


def _spread(n, lo, hi, seed):
    """n lengths between lo and hi, even over their logarithm, as requests of a server differ."""
    rng = np.random.default_rng(seed)
    return _text(int(round(x)) for x in np.exp(rng.uniform(math.log(lo), math.log(hi), n)))


def listed():
    return [
        # a few short prompts, 64-wide heads: launches and latency
        _causal("forward_tiny", "forward", 8, 2, 64, "37,1,90"),
        # the next part of long prompts: fewer queries than keys, three query heads to a K/V head
        _causal("forward_extend", "forward", 24, 8, 128, "256,1,1024,500,77", "5000,301,9000,500,4173"),
        # one long prompt, q, k and v as the projection leaves them in one buffer
        _causal("forward_long", "forward", 32, 8, 128, "32768", packed=True),
        # a small training batch without shared heads
        _causal("step_small", "step", 16, 16, 64, "512,700,129"),
        # a packed training batch of documents
        _causal("step_packed", "step", 32, 8, 128, "4096,1023,2047,877,149"),
        # a training step on long documents, five query heads to a K/V head
        _causal("step_long", "step", 40, 8, 128, "16384,9001"),
        # a serving step of four requests, one new token each
        _tree("tokens_few", 32, 8, 128, 16, "700,64,1500,31", "1,1,1,1"),
        # a serving step of a full batch of uneven requests
        _tree("tokens_batch", 32, 8, 128, 64, _spread(64, 100, 16000, 5), _text([1] * 64)),
        # two requests with very long contexts
        _tree("tokens_long", 32, 8, 128, 32, "131072,120001", "1,1"),
        # drafted trees of up to 48 tokens checked in one pass
        _tree("drafts", 40, 8, 128, 16, _spread(16, 300, 12000, 6), "48,1,17,32,9,48,25,31,40,2,48,16,33,7,21,48"),
        # accepted drafts of a batch go into the cache
        _append("append_drafts", 8, 128, 16, _spread(32, 100, 8000, 7), _spread(32, 1, 8, 8), True),
        # the K/V of whole prompts go into the cache
        _append("append_prompts", 8, 128, 64, "0,4096,0,17", "16384,8192,3001,12345", False),
    ]


def _ints(text):
    return [int(x) for x in text.split(",")]


def _lens(case):
    nq = _ints(case["q_lens"])
    return nq, _ints(case["k_lens"]) if case["k_lens"] else nq


def _pairs(nq, nk):
    """Keys seen by all tokens of one sequence (nq <= nk): i + 1 + nk - nq by token i."""
    return nq * (nk - nq) + nq * (nq + 1) // 2


def work(case):
    if case["op"] in ("forward", "step"):
        nq, nk = _lens(case)
        h, kv, d = case["heads"], case["kv_heads"], case["dim"]
        pairs = sum(_pairs(a, b) for a, b in zip(nq, nk))
        q, k = sum(nq) * h * d * 2, sum(nk) * kv * d * 2
        if case["op"] == "forward":  # in: q, k, v; out: O, LSE
            return {"bytes": 2 * q + 2 * k + sum(nq) * h * 4, "flops": 4 * d * h * pairs}
        # in: q, k, v, dO; out: O, LSE, dQ, dK, dV
        return {"bytes": 4 * q + 4 * k + sum(nq) * h * 4, "flops": 14 * d * h * pairs}
    ctx, new = _ints(case["contexts"]), _ints(case["tokens"])
    row = case["kv_heads"] * case["dim"] * 2
    if case["op"] == "append":
        return {"bytes": 4 * sum(new) * row, "flops": 0}
    h, d = case["heads"], case["dim"]
    seen = sum(t * c + t for c, t in zip(ctx, new))  # at least itself of the drafts
    return {"bytes": 2 * (sum(ctx) + sum(new)) * row + sum(new) * h * (2 * d * 2 + 4), "flops": 4 * d * h * seen}


def draw(rng):
    """One more case: any operator, sizes spread over the logarithm of the range of the listed ones."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["forward", "forward", "step", "step", "tree", "tree", "tree", "append"])
        kv, d = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([64, 128, 128])
        heads = kv * rng.choice([1, 2, 3, 4, 4, 5, 8])
        n = log(1, 12)
        if op in ("forward", "step"):
            longest = log(16, 32768)
            nq = [log(max(1, longest // 8), longest) for _ in range(n)]
            nk = [a + (log(1, 4 * longest) if rng.random() < 0.5 else 0) for a in nq] if rng.random() < 0.3 else nq
            c = _causal(None, op, heads, kv, d, _text(nq), _text(nk) if nk is not nq else "", rng.random() < 0.4)
            if c["packed"] and c["k_lens"]:
                c["packed"] = False
            if work(c)["flops"] > 9.5e12 or sum(nk) * heads * d > 4e8:
                continue
            return c
        n = log(1, 64)
        longest = log(16, 131072)
        ctx = [log(max(1, longest // 16), longest) for _ in range(n)]
        page = rng.choice([8, 16, 16, 32, 64, 128, 256])
        if op == "append":
            picked = rng.random() < 0.5
            most = log(1, 16 if picked else 16384)
            c = _append(None, kv, d, page, _text(ctx), _text(log(max(1, most // 8), most) for _ in ctx), picked)
            if work(c)["bytes"] > 3.2e8 or (sum(ctx) + 128 * n) * kv * d > 5e8:
                continue
            return c
        most = rng.choice([1, 1, log(2, 64)])
        new = [1 if most == 1 else rng.randint(1, most) for _ in ctx]
        c = _tree(None, heads, kv, d, page, _text(ctx), _text(new))
        if heads > 64 or work(c)["bytes"] > 1.05e9 or work(c)["flops"] > 5e11:
            continue
        return c


# ------------------------------------------------------------------------------------------- inputs
def _normal(gen, shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _queries(gen, shape):
    """Queries twice as long: scores of standard deviation 2, so that a row's weight lies on few keys."""
    return 2 * _normal(gen, shape)


def _causal_inputs(case, seed):
    nq, nk = _lens(case)
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["packed"]:  # views of one projection's output
        buf = _normal(gen, (sum(nq), h + 2 * kv, d))
        buf[:, :h] *= 2  # as _queries
        x = {"q": buf[:, :h], "k": buf[:, h:h + kv], "v": buf[:, h + kv:]}
    else:
        x = {"q": _queries(gen, (sum(nq), h, d)), "k": _normal(gen, (sum(nk), kv, d)),
             "v": _normal(gen, (sum(nk), kv, d))}
    if case["op"] == "step":
        x["do"] = _normal(gen, (sum(nq), h, d))
    return x


def _cache_inputs(case, seed):
    """A cache that has served for a while: each sequence's pages lie anywhere in it."""
    ctx, new = _ints(case["contexts"]), _ints(case["tokens"])
    kv, d, page = case["kv_heads"], case["dim"], case["page"]
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    need = [(c + t + page - 1) // page for c, t in zip(ctx, new)]
    pages = sum(need) + 3
    order = rng.permutation(pages)
    table = np.zeros((len(ctx), max(need)), dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)

    def dev(a):
        return torch.from_numpy(a).cuda()

    x = {"k_cache": _normal(gen, (pages, page, kv, d)), "v_cache": _normal(gen, (pages, page, kv, d)),
         "table": dev(table), "context_lens": dev(np.array(ctx, dtype=np.int32)), "cu_tokens": dev(cu)}
    total = int(cu[-1])
    if case["op"] == "append":
        rows = total
        if case["picked"]:  # the accepted ones of four times as many drafts
            rows = 4 * total
            x["rows"] = dev(np.sort(rng.choice(rows, total, replace=False)).astype(np.int32))
        x["k"], x["v"] = _normal(gen, (rows, kv, d)), _normal(gen, (rows, kv, d))
        return x, ctx, new
    x["q"] = _queries(gen, (total, case["heads"], d))
    x["k"], x["v"] = _normal(gen, (total, kv, d)), _normal(gen, (total, kv, d))
    masks = np.zeros(total, dtype=np.uint64)
    for b, t in enumerate(new):  # every draft continues the context or an earlier draft
        for i in range(t):
            parent = int(rng.integers(-1, i)) if i else -1
            above = masks[cu[b] + parent] if parent >= 0 else np.uint64(0)
            masks[cu[b] + i] = above | (np.uint64(1) << np.uint64(i))
    x["tree"] = dev(masks.view(np.int64))
    return x, ctx, new


def prepare(case, seed):
    if case["op"] in ("forward", "step"):
        nq, nk = _lens(case)
        state = {"op": case["op"], "x": _causal_inputs(case, seed), "nq": nq, "nk": nk}
        if own:
            import paper_2606_13872_amd as sra
            state["plan"] = sra.CausalPlan(nq, case["heads"], case["kv_heads"], case["dim"], k_lens=nk,
                                           backward=case["op"] == "step")
        return state
    x, ctx, new = _cache_inputs(case, seed)
    return {"op": case["op"], "x": x, "ctx": ctx, "new": new}


# ------------------------------------------------------------------------------------------ the calls
def run(state):
    if own:
        return _run_own(state)
    return {"forward": _plain_causal, "step": _plain_causal, "tree": _plain_tree, "append": _plain_append}[
        state["op"]](state)


def _run_own(state):
    import paper_2606_13872_amd as sra

    x = state["x"]
    if state["op"] == "append":
        sra.cache_append(x["k"], x["v"], x["k_cache"], x["v_cache"], x["table"], x["context_lens"], x["cu_tokens"],
                         rows=x.get("rows"))
        return {"k_cache": x["k_cache"], "v_cache": x["v_cache"]}
    if state["op"] == "tree":
        o, lse = sra.tree_attention(x["q"], x["k"], x["v"], x["k_cache"], x["v_cache"], x["table"],
                                    x["context_lens"], x["cu_tokens"], tree=x["tree"])
        return {"o": o, "lse": lse}
    o, lse = sra.causal_forward(x["q"], x["k"], x["v"], state["plan"])
    out = {"o": o, "lse": lse}
    if state["op"] == "step":
        out.update(sra.causal_backward(x["q"], x["k"], x["v"], o, lse, x["do"], state["plan"]))
    return out


def _plain_causal(state):
    """Softmax over the scores of every K/V head's query heads, block by block of tokens, in float32."""
    x = state["x"]
    h, d = x["q"].shape[1:]
    kv = x["k"].shape[1]
    g, scale, step = h // kv, 1.0 / math.sqrt(d), state["op"] == "step"
    out = {"o": torch.empty_like(x["q"], memory_format=torch.contiguous_format),
           "lse": torch.empty((h, x["q"].shape[0]), dtype=torch.float32, device="cuda")}
    if step:
        for name, like in (("dq", "q"), ("dk", "k"), ("dv", "v")):
            out[name] = torch.empty_like(x[like], memory_format=torch.contiguous_format)
    q0 = k0 = 0
    for nq, nk in zip(state["nq"], state["nk"]):
        rows = max(1, min(nq, BLOCK // max(1, g * nk)))
        for i in range(kv):
            k, v = x["k"][k0:k0 + nk, i].float(), x["v"][k0:k0 + nk, i].float()
            if step:
                dk, dv = torch.zeros_like(k), torch.zeros_like(v)
            for a in range(0, nq, rows):
                b = min(nq, a + rows)
                n = b + nk - nq  # keys that any of these tokens sees
                at, hs = slice(q0 + a, q0 + b), slice(i * g, (i + 1) * g)
                q = x["q"][at, hs].float().reshape(-1, d)
                s = (q @ k[:n].t()) * scale
                limit = (torch.arange(a, b, device="cuda") + (nk - nq)).repeat_interleave(g)
                s.masked_fill_(torch.arange(n, device="cuda")[None, :] > limit[:, None], -math.inf)
                m = s.amax(-1, keepdim=True)
                e = torch.exp(s - m)
                l = e.sum(-1, keepdim=True)
                p = e / l
                o = p @ v[:n]
                out["o"][at, hs] = o.view(b - a, g, d).to(torch.bfloat16)
                out["lse"][hs, at] = (m + torch.log(l)).view(b - a, g).t()
                if step:
                    do = x["do"][at, hs].float().reshape(-1, d)
                    dv[:n] += p.t() @ do
                    ds = p * (do @ v[:n].t() - (do * o).sum(-1, keepdim=True))
                    out["dq"][at, hs] = ((ds @ k[:n]) * scale).view(b - a, g, d).to(torch.bfloat16)
                    dk[:n] += (ds.t() @ q) * scale
            if step:
                out["dk"][k0:k0 + nk, i], out["dv"][k0:k0 + nk, i] = dk.to(torch.bfloat16), dv.to(torch.bfloat16)
        q0, k0 = q0 + nq, k0 + nk
    return out


def _plain_tree(state):
    x = state["x"]
    h, d = x["q"].shape[1:]
    page, kv = x["k_cache"].shape[1:3]
    g, scale = h // kv, 1.0 / math.sqrt(d)
    o = torch.empty_like(x["q"])
    lse = torch.empty((h, x["q"].shape[0]), dtype=torch.float32, device="cuda")
    t0 = 0
    for b, (c, t) in enumerate(zip(state["ctx"], state["new"])):
        at = slice(t0, t0 + t)
        ids = x["table"][b, :(c + page - 1) // page].long()
        k = torch.cat([x["k_cache"][ids].reshape(-1, kv, d)[:c], x["k"][at]]).float().transpose(0, 1)
        v = torch.cat([x["v_cache"][ids].reshape(-1, kv, d)[:c], x["v"][at]]).float().transpose(0, 1)
        q = x["q"][at].float().reshape(t, kv, g, d).permute(1, 0, 2, 3).reshape(kv, t * g, d)
        s = torch.matmul(q, k.transpose(1, 2)) * scale
        hidden = ((x["tree"][at, None] >> torch.arange(t, device="cuda")) & 1) == 0
        s[:, :, c:].masked_fill_(hidden.repeat_interleave(g, 0)[None], -math.inf)
        m = s.amax(-1, keepdim=True)
        e = torch.exp(s - m)
        l = e.sum(-1, keepdim=True)
        y = torch.matmul(e, v) / l
        o[at] = y.view(kv, t, g, d).permute(1, 0, 2, 3).reshape(t, h, d).to(torch.bfloat16)
        lse[:, at] = (m + torch.log(l)).view(kv, t, g).permute(0, 2, 1).reshape(h, t)
        t0 += t
    return {"o": o, "lse": lse}


def _plain_append(state):
    x = state["x"]
    page = x["k_cache"].shape[1]
    cu = x["cu_tokens"].long()
    token = torch.arange(sum(state["new"]), device="cuda")
    b = torch.searchsorted(cu[1:], token, right=True)
    at = x["context_lens"].long()[b] + token - cu[b]
    ids, slot = x["table"].long()[b, at // page], at % page
    for name in ("k", "v"):
        x[name + "_cache"][ids, slot] = x[name][x["rows"].long()] if "rows" in x else x[name]
    return {"k_cache": x["k_cache"], "v_cache": x["v_cache"]}


# ------------------------------------------------------------------------------------- the definition
def _exact_rows(q, k, v, see, scale):
    """(O, LSE, P) of rows q over k, v in float64, see = which keys each row sees."""
    s = (q @ k.T).mul_(scale)
    s[~see] = -math.inf
    lse = torch.logsumexp(s, -1)
    p = s.sub_(lse[:, None]).exp_()
    return p @ v, lse, p


def _exact_causal(case, seed):
    x = _causal_inputs(case, seed)
    nqs, nks = _lens(case)
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    scale = 1.0 / math.sqrt(d)
    f64 = {"dtype": torch.float64, "device": "cuda"}
    out = {"o": torch.zeros((sum(nqs), h, d), **f64), "lse": torch.zeros((h, sum(nqs)), **f64)}
    if case["op"] == "step":
        out.update(dq=torch.zeros((sum(nqs), h, d), **f64), dk=torch.zeros((sum(nks), kv, d), **f64),
                   dv=torch.zeros((sum(nks), kv, d), **f64))
    q_end = k_end = 0
    for nq, nk in zip(nqs, nks):
        q_end, k_end = q_end + nq, k_end + nk
        for i in range(h):
            j = i * kv // h
            ks = slice(k_end - nk, k_end)
            k, v = x["k"][ks, j].double(), x["v"][ks, j].double()
            key = torch.arange(nk, device="cuda")
            rows = max(1, (1 << 26) // nk)
            for a in range(0, nq, rows):
                b = min(nq, a + rows)
                at = slice(q_end - nq + a, q_end - nq + b)
                # token t of nq stands at position nk - nq + t
                n = nk - nq + b
                see = key[None, :n] <= torch.arange(nk - nq + a, n, device="cuda")[:, None]
                q = x["q"][at, i].double()
                o, lse, p = _exact_rows(q, k[:n], v[:n], see, scale)
                out["o"][at, i], out["lse"][i, at] = o, lse
                if case["op"] == "step":
                    do = x["do"][at, i].double()
                    out["dv"][ks, j][:n] += p.T @ do
                    ds = p.mul_((do @ v[:n].T).sub_((do * o).sum(-1, keepdim=True)))
                    out["dq"][at, i] = scale * (ds @ k[:n])
                    out["dk"][ks, j][:n] += scale * (ds.T @ q)
    return out


def _exact_tree(case, seed):
    x, ctx, new = _cache_inputs(case, seed)
    h, kv, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    f64 = {"dtype": torch.float64, "device": "cuda"}
    out = {"o": torch.zeros((sum(new), h, d), **f64), "lse": torch.zeros((h, sum(new)), **f64)}
    table, tree = x["table"].cpu().numpy(), x["tree"].cpu().numpy().view(np.uint64)
    at = 0
    for b, (c, t) in enumerate(zip(ctx, new)):
        pos = np.arange(c)
        flat = torch.from_numpy(table[b][pos // page].astype(np.int64) * page + pos % page).cuda()
        kc = x["k_cache"].view(-1, kv, d)[flat].double()
        vc = x["v_cache"].view(-1, kv, d)[flat].double()
        see = np.ones((t, c + t), dtype=bool)
        for i in range(t):
            see[i, c:] = [bool(int(tree[at + i]) >> j & 1) for j in range(t)]
        see = torch.from_numpy(see).cuda()
        for i in range(h):
            j = i * kv // h
            k = torch.cat([kc[:, j], x["k"][at:at + t, j].double()])
            v = torch.cat([vc[:, j], x["v"][at:at + t, j].double()])
            o, lse, _ = _exact_rows(x["q"][at:at + t, i].double(), k, v, see, 1.0 / math.sqrt(d))
            out["o"][at:at + t, i], out["lse"][i, at:at + t] = o, lse
        at += t
    return out


def _exact_append(case, seed):
    x, ctx, new = _cache_inputs(case, seed)
    page, table = case["page"], x["table"].cpu().numpy()
    pick = x["rows"].cpu().numpy() if "rows" in x else np.arange(sum(new))
    dst, i = [], 0
    for b, (c, t) in enumerate(zip(ctx, new)):
        dst += [int(table[b, p // page]) * page + p % page for p in range(c, c + t)]
    out = {}
    for name in ("k", "v"):
        cache = x[name + "_cache"].double()
        cache.view(-1, *cache.shape[2:])[torch.tensor(dst, device="cuda")] = x[name][
            torch.from_numpy(pick).cuda().long()].double()
        out[name + "_cache"] = cache
    return out


def exact(case, seed):
    if work(case)["flops"] > 2e13:
        return None
    if case["op"] == "tree":
        return _exact_tree(case, seed)
    return _exact_append(case, seed) if case["op"] == "append" else _exact_causal(case, seed)
