"""Plain float64 definitions of the language-model operators (causal attention of packed prompts, attention of drafted
tokens over a paged cache, appending to it), with the error bounds that their bf16 roundings allow.

Test infrastructure only; it shares no code with the HIP path. Torch tensors on any device, float64 throughout.

Bounds. With u = 2^-8, half a step of bf16: P is rounded to bf16 before P V, and O when it is stored, so
|O error| <= u (|O| + sum_j P_j |V_j|) elementwise. In the backward P (for dV) and dS (for dQ and dK) are rounded, and
the results when they are stored; D = rowsum(dO * O) takes the stored O, so dS is off by u |dS| + P |D error|. The
32-bit sums, products and exponentials add less than a hundredth of that where |scores| stay below 100, except for
a score's own error, at most e = head_dim 2^-24 scale sum_c |q_c k_c|, which is a relative error of its P (SLACK
and the term `e`). The log-sum-exp has that error alone.
"""
import math

import torch

U = 2.0 ** -8
SLACK = 1.05  # of the bounds, for the 32-bit roundings


def causal_mask(nq, nk, device="cpu"):
    """see[i, j]: token i of nq sees key j of nk, j <= i + nk - nq."""
    i = torch.arange(nq, device=device)[:, None]
    return torch.arange(nk, device=device)[None, :] <= i + (nk - nq)


def _score_error(q, k, scale):
    """Largest error of a row's scores (32-bit sums of exact products), per row."""
    if k.shape[0] == 0:
        return torch.zeros(q.shape[0], dtype=q.dtype, device=q.device)
    return q.shape[1] * 2.0 ** -24 * scale * (q.abs() @ k.abs().T).amax(-1)


def rows(q, k, v, see, scale):
    """Softmax attention of rows q over k, v where see: o, lse, P and the bounds of o and lse."""
    s = (q @ k.T) * scale
    s = torch.where(see, s, -math.inf)
    some = see.any(-1)
    m = torch.where(some, s.amax(-1) if k.shape[0] else torch.zeros_like(some, dtype=q.dtype), 0.0)
    e = torch.exp(s - m[:, None])
    l = e.sum(-1)
    p = e / torch.where(some, l, 1.0)[:, None]
    lse = torch.where(some, m + torch.log(l), -math.inf)
    o = p @ v
    err = _score_error(q, k, scale)
    o_err = SLACK * (U * (o.abs() + p @ v.abs()) + 2 * err[:, None] * (p @ v.abs())) + 1e-30
    lse_err = err + 1e-6 + 2.0 ** -22 * torch.where(some, lse.abs(), 0.0)
    return o, lse, p, o_err, lse_err


def row_gradients(q, k, v, do, o, p, o_err, scale):
    """dq, dk, dv of rows() with upstream do, and their bounds, before the results are stored."""
    d = (do * o).sum(-1, keepdim=True)
    d_err = (do.abs() * o_err).sum(-1, keepdim=True)
    dv = p.T @ do
    ds = p * (do @ v.T - d)
    err = 2 * _score_error(q, k, scale)[:, None]
    ds_err = (U + err) * ds.abs() + p * d_err
    dq, dk = scale * (ds @ k), scale * (ds.T @ q)
    return (dq, dk, dv), (scale * (ds_err @ k.abs()), scale * (ds_err.T @ q.abs()),
                          (p * (U + err)).T @ do.abs())


def causal(q, k, v, q_lens, k_lens, scale=None, do=None):
    """Values and bounds of causal attention: dicts o, lse and, with do, dq, dk, dv."""
    q, k, v = q.double(), k.double(), v.double()
    do = None if do is None else do.double()
    h, d = q.shape[1:]
    g = h // k.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    names = ["o", "dq"] if do is not None else ["o"]
    val = {n: torch.zeros_like(q) for n in names}
    val["lse"] = torch.full((h, q.shape[0]), -math.inf, dtype=q.dtype, device=q.device)
    if do is not None:
        val.update(dk=torch.zeros_like(k), dv=torch.zeros_like(v))
    bound = {n: torch.zeros_like(t) for n, t in val.items()}
    q0 = k0 = 0
    for nq, nk in zip(q_lens, k_lens):
        qs, ks = slice(q0, q0 + nq), slice(k0, k0 + nk)
        q0, k0 = q0 + nq, k0 + nk
        if nq == 0:
            continue
        see = causal_mask(nq, nk, q.device)
        for i in range(h):
            kk, vv, qq = k[ks, i // g], v[ks, i // g], q[qs, i]
            o, lse, p, o_err, lse_err = rows(qq, kk, vv, see, scale)
            val["o"][qs, i], bound["o"][qs, i] = o, o_err
            val["lse"][i, qs], bound["lse"][i, qs] = lse, lse_err
            if do is None:
                continue
            (dq, dk, dv), (eq, ek, ev) = row_gradients(qq, kk, vv, do[qs, i], o, p, o_err, scale)
            val["dq"][qs, i], bound["dq"][qs, i] = dq, eq
            val["dk"][ks, i // g] += dk
            bound["dk"][ks, i // g] += ek
            val["dv"][ks, i // g] += dv
            bound["dv"][ks, i // g] += ev
    for n in ("dq", "dk", "dv"):
        if n in val:
            bound[n] = SLACK * (bound[n] + U * val[n].abs()) + 1e-30
    return val, bound


def within(got, want, bound):
    """(whether every element of got lies within its bound of want, the largest error in bounds)."""
    got = got.double()
    same = (got == want)  # infinities
    err = torch.where(same, torch.zeros_like(want), (got - want).abs() / bound)
    err = torch.where(torch.isnan(err), torch.full_like(err, math.inf), err)
    worst = float(err.max()) if err.numel() else 0.0
    return worst <= 1.0, worst


def gather_cache(cache, table_row, n):
    """The first n rows of a sequence in cache [pages, page_size, heads, dim], in order."""
    page = cache.shape[1]
    pos = torch.arange(n, device=cache.device)
    return cache[table_row.long()[pos // page], pos % page]


def tree(q, k, v, k_cache, v_cache, table, context_lens, cu_tokens, masks=None, scale=None):
    """Values and bounds (o, lse) of drafted tokens over their context and each other.
    masks: ints, bit j of token i = it sees drafted token j of its sequence; None = all up to itself.
    Rows of tokens outside every sequence are NaN in the values."""
    q, k, v = q.double(), k.double(), v.double()
    h, d = q.shape[1:]
    kv = k.shape[1]
    g = h // kv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    val = {"o": torch.full_like(q, math.nan), "lse": torch.full((h, q.shape[0]), math.nan, dtype=q.dtype, device=q.device)}
    bound = {n: torch.ones_like(t) for n, t in val.items()}
    for b, c in enumerate(context_lens):
        t0, t1 = cu_tokens[b], cu_tokens[b + 1]
        t = t1 - t0
        if t == 0:
            continue
        kc = gather_cache(k_cache, table[b], c).double()
        vc = gather_cache(v_cache, table[b], c).double()
        see = torch.ones((t, c + t), dtype=torch.bool)
        for i in range(t):
            for j in range(t):
                see[i, c + j] = (j <= i) if masks is None else (j < 64 and bool((int(masks[t0 + i]) >> j) & 1))
        see = see.to(q.device)
        for i in range(h):
            kk, vv = torch.cat([kc[:, i // g], k[t0:t1, i // g]]), torch.cat([vc[:, i // g], v[t0:t1, i // g]])
            o, lse, _, o_err, lse_err = rows(q[t0:t1, i], kk, vv, see, scale)
            val["o"][t0:t1, i], bound["o"][t0:t1, i] = o, o_err
            val["lse"][i, t0:t1], bound["lse"][i, t0:t1] = lse, lse_err
    return val, bound
