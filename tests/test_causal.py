"""Causal attention of packed prompts on the host: the plan's tables against the rule, the float64 definition against
itself, and every refusal."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

import paper_2606_13872_amd as sra
from oracle import text_oracle as T
from paper_2606_13872_amd import causal as binding


@pytest.mark.parametrize("nq,nk", [([1], [1]), ([37, 1, 90], [37, 1, 90]), ([700, 0, 5], [900, 10, 3]), ([40, 300], [0, 1]),
                                   ([257], [257]), ([3000], [3000]), ([64, 2100], [64, 4100]), ([5], [600])])
@pytest.mark.parametrize("heads,kv", [(8, 2), (3, 3), (6, 2), (7, 1)])
def test_plan_covers_exactly_the_causal_mask(nq, nk, heads, kv):
    plan = sra.CausalPlan(nq, heads, kv, 64, k_lens=nk)
    for b, which, h in itertools.product(range(len(nq)), range(3), sorted({0, heads // 2, heads - 1})):
        want = T.causal_mask(nq[b], nk[b]).numpy().astype(np.uint8)
        got = plan.mask(which, b, h)
        assert got.shape == want.shape and np.array_equal(got, want), (b, which, h)


def test_long_launches_cover_exactly_the_causal_mask_in_larger_items():
    nq = [900, 385, 1] + [5] * 300
    for d in (64, 128):
        plan = sra.CausalPlan(nq, 16, 8, d)
        assert plan.forward_workspace == 0
        for b, which, h in itertools.product((0, 1, 2, 200), range(3), (0, 15)):
            assert np.array_equal(plan.mask(which, b, h), T.causal_mask(nq[b], nq[b]).numpy().astype(np.uint8))


def test_long_items_of_short_launches_are_split_and_sizes_follow():
    whole = sra.CausalPlan([128] * 64, 8, 8, 128)
    assert whole.forward_workspace == 0
    cut = sra.CausalPlan([8192], 2, 1, 128)
    assert cut.forward_workspace > 0 and cut.backward_workspace > 2 * 2 * 8192 * 4
    assert sra.CausalPlan([8192], 2, 1, 128, backward=False).backward_workspace == 0


def test_definition_matches_differences():
    """The float64 gradients against central differences of the float64 forward."""
    g = torch.Generator().manual_seed(0)
    nq, nk = [5, 3], [7, 2]
    q, do = (torch.randn(8, 4, 8, generator=g, dtype=torch.float64) for _ in range(2))
    k, v = (torch.randn(9, 2, 8, generator=g, dtype=torch.float64) for _ in range(2))
    val, _ = T.causal(q, k, v, nq, nk, do=do)

    def loss(**x):
        a = {"q": q, "k": k, "v": v, **x}
        return float((T.causal(a["q"], a["k"], a["v"], nq, nk)[0]["o"] * do).sum())

    for name, t, grad in (("q", q, "dq"), ("k", k, "dk"), ("v", v, "dv")):
        for i in torch.randint(0, t.numel(), (12,), generator=g).tolist():
            lo, hi = t.clone(), t.clone()
            lo.view(-1)[i] -= 1e-5
            hi.view(-1)[i] += 1e-5
            # central differences: h^2 ~ 1e-10 of the third derivative, rounding ~ 1e-16 / 1e-5
            assert abs((loss(**{name: hi}) - loss(**{name: lo})) / 2e-5 - float(val[grad].view(-1)[i])) < 1e-8


def test_definition_matches_library_softmax():
    g = torch.Generator().manual_seed(1)
    q = torch.randn(40, 2, 16, generator=g, dtype=torch.float64)
    k, v = (torch.randn(40, 1, 16, generator=g, dtype=torch.float64) for _ in range(2))
    val, bound = T.causal(q, k, v, [40], [40])
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), k.transpose(0, 1).expand(2, -1, -1),
                                                            v.transpose(0, 1).expand(2, -1, -1), is_causal=True)
    assert float((val["o"] - want.transpose(0, 1)).abs().max()) < 1e-12
    assert T.within(val["o"], val["o"], bound["o"])[0]
    off = val["o"].clone()
    off[39, 0, 0] += 0.2 * off.abs().max()  # a planted mistake in one element
    assert not T.within(off, val["o"], bound["o"])[0]


@pytest.mark.parametrize("args,status", [
    (dict(q_lens=[], heads=4, kv_heads=2, head_dim=64), 1), (dict(q_lens=[-1], heads=4, kv_heads=2, head_dim=64), 1),
    (dict(q_lens=[1.5], heads=4, kv_heads=2, head_dim=64), 1), (dict(q_lens=[[4]], heads=4, kv_heads=2, head_dim=64), 1),
    (dict(q_lens=[2**31], heads=4, kv_heads=2, head_dim=64), 1),
    (dict(q_lens=[4], heads=4, kv_heads=2, head_dim=64, k_lens=[4, 4]), 1),
    (dict(q_lens=[4], heads=4, kv_heads=2, head_dim=64, k_lens=[-4]), 1),
    (dict(q_lens=[4], heads=4, kv_heads=3, head_dim=64), 1), (dict(q_lens=[4], heads=0, kv_heads=1, head_dim=64), 1),
    (dict(q_lens=[4], heads=2, kv_heads=0, head_dim=64), 1), (dict(q_lens=[4], heads=2, kv_heads=4, head_dim=64), 1),
    (dict(q_lens=[4], heads=4, kv_heads=2, head_dim=0), 1), (dict(q_lens=[4], heads=4, kv_heads=2, head_dim=96), 2),
    (dict(q_lens=[2**30, 2**30], heads=1, kv_heads=1, head_dim=64), 2),   # 2^31 rows
    (dict(q_lens=[1], heads=2, kv_heads=2, head_dim=64, k_lens=[2**30]), 2),
])
def test_bad_plans_are_refused(args, status):
    with pytest.raises(sra.SRAError) as e:
        sra.CausalPlan(**args)
    assert e.value.status == status


def _args(plan, device="cpu"):
    bf = torch.bfloat16
    q = torch.zeros(plan.n_q, plan.heads, plan.head_dim, dtype=bf, device=device)
    k = torch.zeros(plan.n_k, plan.kv_heads, plan.head_dim, dtype=bf, device=device)
    return q, k, k.clone()


def test_bad_tensors_are_refused_before_anything_reaches_the_library():
    plan = sra.CausalPlan([30, 4], 4, 2, 64)
    q, k, v = _args(plan)
    lse = torch.zeros(4, 34)
    bad = {
        "dtype": lambda: sra.causal_forward(q.float(), k, v, plan),
        "q shape": lambda: sra.causal_forward(q[:-1], k, v, plan),
        "k heads": lambda: sra.causal_forward(q, q, v, plan),
        "v shape": lambda: sra.causal_forward(q, k, v[1:], plan),
        "head layout": lambda: sra.causal_forward(q.transpose(0, 1).contiguous().transpose(0, 1), k, v, plan),
        "overlapping tokens": lambda: sra.causal_forward(q, k[:1].expand(34, 2, 64), v, plan),
        "not a plan": lambda: sra.causal_forward(q, k, v, [30, 4]),
        "not a tensor": lambda: sra.causal_forward(q, k, None, plan),
        "cpu tensors": lambda: sra.causal_forward(q, k, v, plan),
        "out dtype": lambda: sra.causal_forward(q, k, v, plan, out={"o": q.float()}),
        "out layout": lambda: sra.causal_forward(q, k, v, plan, out={"lse": torch.zeros(34, 4).t()}),
        "lse shape": lambda: sra.causal_backward(q, k, v, q, lse[:, :-1], q, plan),
        "do dtype": lambda: sra.causal_backward(q, k, v, q, lse, q.float(), plan),
        "backward on cpu": lambda: sra.causal_backward(q, k, v, q, lse, q, plan),
        "forward-only plan": lambda: sra.causal_backward(q, k, v, q, lse, q, sra.CausalPlan([30, 4], 4, 2, 64, backward=False)),
    }
    for name, call in bad.items():
        with pytest.raises(sra.SRAError) as e:
            call()
        assert e.value.status == 1, name


def test_outputs_that_overlap_inputs_are_found():
    t = torch.zeros(100, 2, 64, dtype=torch.bfloat16)
    binding._no_alias({}, (("q", t), ("k", t)))  # inputs may share memory
    binding._no_alias({"o": 1}, (("q", t[:50]), ("o", t[50:])))
    for out in ({"o": 1}, {"o": 1, "q2": 1}):
        with pytest.raises(sra.SRAError):
            binding._no_alias(out, (("q", t), ("o", t[50:])))


def test_library_refuses_before_any_launch():
    plan = sra.CausalPlan([300], 4, 2, 64)
    L, h = binding._lib(), plan._handle
    fake, null = ctypes.c_void_p(1 << 20), ctypes.c_void_p(0)

    def fwd(handle=h, tables=fake, q=fake, k=fake, o=fake, qs=0, ks=0, scale=0.0, ws=fake, n=1 << 30):
        return L.sra_causal_forward(handle, tables, q, k, fake, qs, ks, 0, o, fake, scale, ws, n, null)

    odd = ctypes.c_void_p((1 << 20) + 2)
    assert fwd(handle=null) == 1 and fwd(tables=null) == 1 and fwd(tables=odd) == 1
    assert fwd(q=null) == 1 and fwd(k=odd) == 1 and fwd(o=null) == 1
    assert fwd(qs=128) == 1 and fwd(qs=260) == 1 and fwd(ks=64) == 1 and fwd(ks=1 << 40) == 2
    assert fwd(scale=float("nan")) == 1 and fwd(scale=float("inf")) == 1
    cut = sra.CausalPlan([8192], 2, 1, 128)
    args = (cut._handle, fake, fake, fake, fake, 0, 0, 0, fake, fake, 0.0)
    assert L.sra_causal_forward(*args, fake, cut.forward_workspace - 1, null) == 3
    assert L.sra_causal_forward(*args, odd, cut.forward_workspace, null) == 1
    only = sra.CausalPlan([300], 4, 2, 64, backward=False)
    bargs = (fake, fake, fake, fake, 0, 0, 0, fake, fake, fake, fake, fake, fake, 0.0)
    assert L.sra_causal_backward(only._handle, *bargs, fake, 1 << 30, null) == 1
    assert L.sra_causal_backward(h, *bargs, fake, plan.backward_workspace - 256, null) == 3
    assert len(L.sra_last_error()) > 0
    assert L.sra_causal_plan_tables(h, null, plan._table_bytes) == 1
    assert L.sra_causal_plan_mask(h, 7, 0, 0, fake) == 1 and L.sra_causal_plan_mask(h, 0, 1, 0, fake) == 1
    assert L.sra_causal_plan_destroy(null) == 0


@pytest.mark.parametrize("args", [
    dict(q_lens=[2**28], heads=1, kv_heads=1, head_dim=64), dict(q_lens=[1], k_lens=[2**24], heads=32, kv_heads=16, head_dim=64),
    dict(q_lens=[2**31 - 1] * 4, heads=2**30, kv_heads=2**30, head_dim=64),  # their product passes 64 bits
    dict(q_lens=[0], heads=2**24, kv_heads=1, head_dim=64), dict(q_lens=[0, 1] * 2**15, heads=256, kv_heads=256, head_dim=128),
])
def test_sizes_past_what_a_launch_takes_are_refused(args):
    with pytest.raises(sra.SRAError) as e:
        sra.CausalPlan(**args)
    assert e.value.status == 2


def test_largest_plans():
    p = sra.CausalPlan([1], 1, 1, 64, k_lens=[2**28 - 1])
    assert p.n_k == 2**28 - 1 and p.backward_workspace > 0
    assert sra.CausalPlan([2**18 - 1], 1, 1, 128, k_lens=[1], backward=False).n_q == 2**18 - 1


def _longest_items(plan):
    """Rows or keys of the longest item of each kind in the plan's tables (records of 12 int32, sections 256-byte aligned)."""
    t = np.zeros(plan._table_bytes, dtype=np.uint8)
    assert binding._lib().sra_causal_plan_tables(plan._handle, t.ctypes.data, plan._table_bytes) == 0
    r, at, longest = t.view(np.int32), 0, {0: 0, 1: 0, 2: 0}
    while at + 12 <= len(r):
        if r[at + 3] > 0:
            longest[int(r[at])] = max(longest[int(r[at])], int(r[at + 3]))
            at += 12
        else:
            at = (at // 64 + 1) * 64
    return longest


@pytest.mark.parametrize("lens,heads,kv,d,forward,cut,backward", [
    ([700], 4, 2, 128, 128, False, 128), ([2500, 311], 2, 2, 64, 128, True, 256), ([2000, 1900, 300], 24, 8, 128, 256, False, 256),
    ([1500, 200, 900] * 3, 16, 8, 64, 256, False, 256), ([4099], 4, 1, 128, 256, True, 256), ([4099], 4, 1, 64, 256, True, 256),
    ([1500, 200, 900] * 3, 16, 8, 128, 384, False, 256), ([9000] * 2, 32, 8, 64, 512, False, 256),
])
def test_items_grow_with_the_launch(lens, heads, kv, d, forward, cut, backward):
    p = sra.CausalPlan(lens, heads, kv, d)
    n = _longest_items(p)
    assert (n[0], n[1], n[2]) == (forward, backward, backward) and (p.forward_workspace > 0) == cut
