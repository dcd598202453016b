"""Causal attention of packed prompts on the GPU against its float64 definition, within the bounds of its
roundings (oracle/text_oracle.py)."""
import pytest
import torch

import paper_2606_13872_amd as sra
from oracle import text_oracle as T

pytestmark = pytest.mark.gpu


def _inputs(nq, nk, heads, kv, d, seed=0, size=1.0, packed=False):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    q, k, v, do = normal(sum(nq), heads, d) * size, normal(sum(nk), kv, d), normal(sum(nk), kv, d), normal(sum(nq), heads, d)
    q, k, v, do = (t.to(torch.bfloat16) for t in (q, k, v, do))
    if packed:
        assert nq == nk
        buf = torch.cat([q, k, v], dim=1)
        q, k, v = buf[:, :heads], buf[:, heads:heads + kv], buf[:, heads + kv:]
    return q, k, v, do


def _check(nq, nk, heads, kv, d, scale=None, **kw):
    q, k, v, do = _inputs(nq, nk, heads, kv, d, **kw)
    plan = sra.CausalPlan(nq, heads, kv, d, k_lens=nk)
    o, lse = sra.causal_forward(q, k, v, plan, scale=scale)
    got = {"o": o, "lse": lse, **sra.causal_backward(q, k, v, o, lse, do, plan, scale=scale)}
    val, bound = T.causal(q, k, v, nq, nk, scale=scale, do=do)
    for n in val:
        ok, worst = T.within(got[n], val[n], bound[n])
        assert ok, f"{n}: {worst:.2f} bounds off"
        # One step of bf16 is 0.004 of a value, roundings add up as their squares. (A row that sees one key has P = 1
        # and D = dO V, so its dS, dQ and dK are 0 and no error is small beside them: tensors made of such rows, whose
        # bounds exceed their values, have the bounds alone.)
        if n != "lse" and float(bound[n].norm()) < float(val[n].norm()):
            rel = float((got[n].double() - val[n]).norm() / val[n].norm().clamp(min=1e-30))
            assert rel <= 1e-2, f"{n}: relative error {rel:.2e}"
    return got


LENGTHS = [
    ([1], [1]),
    ([37, 1, 90], [37, 1, 90]),
    ([64, 65, 63, 128, 256, 257], [64, 65, 63, 128, 256, 257]),
    ([700, 0, 5, 33], [900, 10, 3, 95]),       # continued sequences, one without tokens, one with empty rows
    ([40, 300], [0, 1]),                       # no keys at all; rows that see nothing
    ([1, 1, 1], [1000, 64, 65]),               # single tokens behind long contexts
    ([1030], [1030]),
]


@pytest.mark.parametrize("nq,nk", LENGTHS)
@pytest.mark.parametrize("heads,kv,d", [(8, 2, 64), (4, 4, 128), (6, 2, 128), (5, 1, 64), (16, 1, 128)])
def test_forward_and_gradients(nq, nk, heads, kv, d):
    print("causal", nq, nk, heads, kv, d, flush=True)
    _check(nq, nk, heads, kv, d, seed=sum(nq) + heads)


@pytest.mark.parametrize("d", [64, 128])
def test_long_sequences(d):
    """Splits of long items (one sequence, few heads) and several rounds of the pipelined loop."""
    print("causal long", d, flush=True)
    _check([4099], [4099], 4, 1, d, seed=3)
    _check([2500, 311], [4000, 311], 2, 2, d, seed=4)


@pytest.mark.parametrize("heads,kv,d", [(16, 8, 128), (8, 8, 64)])
def test_many_sequences(heads, kv, d):
    """Launches too long to be cut: the larger forward items, dK/dV and dQ one after the other."""
    print("causal many", heads, kv, d, flush=True)
    nq = [900, 385, 1, 513] + [3, 17] * 150
    nk = [900, 500, 1, 600] + [3, 17] * 150
    assert sum(-(-n * (heads // kv) // 256) for n in nq) * kv > 2048
    _check(nq, nk, heads, kv, d, seed=15)


@pytest.mark.parametrize("size,scale", [(3.0, None), (1.0, 1.0), (1.0, 0.02)])
def test_peaked_and_flat_scores(size, scale):
    """Scores whose running maximum keeps rising, and custom scales."""
    print("causal scores", size, scale, flush=True)
    _check([900, 130], [900, 130], 4, 2, 128, seed=5, size=size, scale=scale)
    _check([900, 130], [900, 130], 4, 2, 64, seed=6, size=size, scale=scale)


@pytest.mark.parametrize("d", [64, 128])
def test_views_of_one_buffer(d):
    print("causal packed", d, flush=True)
    _check([300, 77, 512], [300, 77, 512], 8, 2, d, seed=7, packed=True)


def test_separate_strides_of_k_and_v():
    print("causal strides", flush=True)
    nq = [200, 65]
    q, k, v, do = _inputs(nq, nq, 4, 2, 128, seed=8)
    kw = torch.zeros(265, 5, 128, dtype=torch.bfloat16, device="cuda")
    kw[:, 1:3] = k
    vw = torch.zeros(265, 3, 128, dtype=torch.bfloat16, device="cuda")
    vw[:, 1:] = v
    plan = sra.CausalPlan(nq, 4, 2, 128)
    a = sra.causal_forward(q, k, v, plan)
    b = sra.causal_forward(q, kw[:, 1:3], vw[:, 1:], plan)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ga = sra.causal_backward(q, k, v, *a, do, plan)
    gb = sra.causal_backward(q, kw[:, 1:3], vw[:, 1:], *a, do, plan)
    for n in ga:
        assert torch.equal(ga[n], gb[n]), n


def test_future_tokens_and_other_sequences_do_not_reach_a_row():
    """Bitwise: a token's row does not change with later tokens, nor with other sequences' (even infinite ones)."""
    print("causal future", flush=True)
    nq = [300, 200]
    q, k, v, _ = _inputs(nq, nq, 4, 2, 128, seed=9)
    plan = sra.CausalPlan(nq, 4, 2, 128, backward=False)
    o, lse = sra.causal_forward(q, k, v, plan)
    k2, v2 = k.clone(), v.clone()
    k2[150:300], v2[150:300] = 7.0, -3.0
    k2[300:], v2[300:] = float("inf"), float("nan")
    o2, lse2 = sra.causal_forward(q, k2, v2, plan)
    assert torch.equal(o[:150], o2[:150]) and torch.equal(lse[:, :150], lse2[:, :150])
    assert not torch.equal(o[200:300], o2[200:300]) and bool(torch.isfinite(o2[:300].float()).all())


def test_empty_rows():
    print("causal empty rows", flush=True)
    nq, nk = [90, 3], [20, 0]
    got = _check(nq, nk, 4, 2, 64, seed=10)
    assert bool((got["o"][:70] == 0).all()) and bool((got["lse"][:, :70] == -float("inf")).all())
    assert bool((got["dq"][:70] == 0).all()) and bool((got["o"][90:] == 0).all())


def test_no_tokens_and_no_keys():
    print("causal nothing", flush=True)
    got = _check([0], [70], 4, 2, 128)
    assert got["o"].shape == (0, 4, 128) and bool((got["dk"] == 0).all()) and bool((got["dv"] == 0).all())
    got = _check([3, 0], [0, 0], 4, 2, 64)
    assert bool((got["lse"] == -float("inf")).all()) and bool((got["dq"] == 0).all()) and got["dk"].numel() == 0


def test_kernel_timing_counts_the_launches():
    print("causal timing", flush=True)
    q, k, v, do = _inputs([300], [300], 4, 2, 64)
    plan = sra.CausalPlan([300], 4, 2, 64)
    sra.sra.kernel_timing_enable(True)
    for _ in range(3):
        o, lse = sra.causal_forward(q, k, v, plan)
    sra.causal_backward(q, k, v, o, lse, do, plan)
    t = sra.sra.kernel_timing()
    sra.sra.kernel_timing_enable(False)
    assert t["causal_forward"][1] == 3 and t["causal_delta"][1] == 1 and t["causal_grad"][1] == 1 and t["forward"][1] == 0
    assert all(t[n][0] > 0 for n in ("causal_forward", "causal_delta", "causal_grad"))


def test_repeats_are_bitwise_equal_and_buffers_are_used():
    print("causal repeats", flush=True)
    nq = [777, 130]
    q, k, v, do = _inputs(nq, nq, 6, 3, 128, seed=11)
    plan = sra.CausalPlan(nq, 6, 3, 128)
    o, lse = sra.causal_forward(q, k, v, plan)
    g = sra.causal_backward(q, k, v, o, lse, do, plan)
    out = {"o": torch.full_like(o, 9), "lse": torch.full_like(lse, 9),
           "workspace": torch.empty(max(plan.backward_workspace, plan.forward_workspace), dtype=torch.uint8, device="cuda")}
    o2, lse2 = sra.causal_forward(q, k, v, plan, out=out)
    assert o2 is out["o"] and lse2 is out["lse"]
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    gout = {n: torch.full_like(t, 9) for n, t in g.items()}
    g2 = sra.causal_backward(q, k, v, o, lse, do, plan, out={**gout, "workspace": out["workspace"]})
    for n in g:
        assert g2[n] is gout[n] and torch.equal(g[n], g2[n]), n


def test_writes_stay_inside_the_outputs():
    print("causal guards", flush=True)
    nq, nk = [257, 31], [300, 31]
    q, k, v, do = _inputs(nq, nk, 4, 2, 64, seed=12)
    plan = sra.CausalPlan(nq, 4, 2, 64, k_lens=nk)

    def guarded(shape, dtype):
        n = 1
        for s in shape:
            n *= s
        buf = torch.full((n + 2048,), 123.0, dtype=dtype, device="cuda")
        return buf, buf[1024:1024 + n].view(shape)

    bufs = {n: guarded(s, t) for n, s, t in (("o", q.shape, torch.bfloat16), ("lse", (4, 288), torch.float32),
                                             ("dq", q.shape, torch.bfloat16), ("dk", k.shape, torch.bfloat16),
                                             ("dv", k.shape, torch.bfloat16))}
    o, lse = sra.causal_forward(q, k, v, plan, out={n: bufs[n][1] for n in ("o", "lse")})
    sra.causal_backward(q, k, v, o, lse, do, plan, out={n: bufs[n][1] for n in ("dq", "dk", "dv")})
    for n, (buf, t) in bufs.items():
        assert bool((buf[:1024] == 123).all()) and bool((buf[1024 + t.numel():] == 123).all()), n


def test_captured_calls_replay():
    """Both directions in one graph, replayed on new inputs, with eager calls of another plan in between."""
    print("causal graph", flush=True)
    nq = [600, 77]
    q, k, v, do = _inputs(nq, nq, 4, 1, 128, seed=13)
    plan, other = sra.CausalPlan(nq, 4, 1, 128), sra.CausalPlan([50, 1000], 4, 1, 128)
    sra.causal_forward(q, k, v, plan)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = sra.causal_forward(q, k, v, plan)
        g = sra.causal_backward(q, k, v, o, lse, do, plan)
    for seed in (20, 21, 22):
        for dst, src in zip((q, k, v, do), _inputs(nq, nq, 4, 1, 128, seed=seed)):
            dst.copy_(src)
        graph.replay()
        x = _inputs([50, 1000], [50, 1000], 4, 1, 128, seed=seed)
        sra.causal_forward(*x[:3], other)
        torch.cuda.synchronize()
        o2, lse2 = sra.causal_forward(q, k, v, plan)
        g2 = sra.causal_backward(q, k, v, o2, lse2, do, plan)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        for n in g:
            assert torch.equal(g[n], g2[n]), n


def test_two_streams_at_once():
    print("causal streams", flush=True)
    nq = [1500]
    q, k, v, do = _inputs(nq, nq, 4, 2, 128, seed=14)
    plan = sra.CausalPlan(nq, 4, 2, 128)
    o, lse = sra.causal_forward(q, k, v, plan)
    want = sra.causal_backward(q, k, v, o, lse, do, plan)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    res = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                a = sra.causal_forward(q, k, v, plan)
                res.append((a, sra.causal_backward(q, k, v, *a, do, plan)))
    torch.cuda.synchronize()
    for a, g in res:
        assert torch.equal(a[0], o) and torch.equal(a[1], lse)
        for n in g:
            assert torch.equal(g[n], want[n]), n


def test_plans_are_made_outside_a_capture():
    x = torch.zeros(1, device="cuda")
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(sra.SRAError, match="capture"):
            sra.CausalPlan([5], 4, 2, 64)
        x.add_(1)


@pytest.mark.parametrize("nq,nk,heads,kv,d", [
    ([2000, 1900, 300], [2000, 1900, 300], 24, 8, 128), ([1500, 200, 900] * 3, [1500, 200, 900] * 3, 16, 8, 64),
    ([1500, 200, 900] * 3, [1500, 200, 900] * 3, 16, 8, 128), ([1800, 77, 1100], [2300, 77, 1500], 40, 8, 128),
    ([2500, 311], [2500, 311], 2, 2, 64),
])
def test_launches_between_short_and_long(nq, nk, heads, kv, d):
    """Items of 256 rows that are not cut, cut ones of 128, and their neighbours."""
    print("causal middle", nq, heads, kv, d, flush=True)
    _check(nq, nk, heads, kv, d, seed=40 + heads)
