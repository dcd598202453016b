"""What one packed sequence holds does not reach another's outputs or gradients, on the GPU, bitwise; and wide groups of heads."""
import math

import pytest
import torch

import paper_2606_13872_amd as sra
from test_gpu_causal import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq,nk,heads,kv", [
    ([70, 65, 1, 130, 255], [70, 65, 1, 130, 255], 4, 1),       # next to the tiles' edges
    ([63, 31, 2, 200], [90, 31, 65, 257], 6, 2),                # keys that precede the queries
    ([2500, 33, 300], [2500, 33, 300], 2, 2),                   # long items in pieces
    ([5, 40, 300], [2, 0, 301], 4, 4),                          # rows that see nothing, no keys
    ([900, 3, 17] + [5] * 260, [900, 3, 17] + [5] * 260, 16, 8),  # a launch that is not cut
])
@pytest.mark.parametrize("d", [64, 128])
def test_infinities_and_nan_stay_in_their_sequence(nq, nk, heads, kv, d):
    print("causal poison", nq[:5], heads, kv, d, flush=True)
    q, k, v, do = _inputs(nq, nk, heads, kv, d, seed=16)
    plan = sra.CausalPlan(nq, heads, kv, d, k_lens=nk)

    def step(q, k, v, do):
        o, lse = sra.causal_forward(q, k, v, plan)
        return {"o": o, "lse": lse.t(), **sra.causal_backward(q, k, v, o, lse, do, plan)}

    want = step(q, k, v, do)
    for b in range(min(len(nq), 5)):
        qs, ks = (slice(sum(n[:b]), sum(n[:b + 1])) for n in (nq, nk))
        for bad in (math.inf, -math.inf, math.nan):
            x = [t.clone() for t in (q, k, v, do)]
            for t, at in zip(x, (qs, ks, ks, qs)):
                t[at] = bad
            got = step(*x)
            for n, t in want.items():
                keep = torch.ones(t.shape[0], dtype=torch.bool, device="cuda")
                keep[ks if n in ("dk", "dv") else qs] = False
                assert torch.equal(got[n][keep], t[keep]), (n, b, bad)


@pytest.mark.parametrize("heads,kv,d,nq,nk", [(300, 1, 64, [5, 70], [9, 70]), (99, 3, 128, [65, 2], [65, 300])])
def test_many_heads_of_one_key_head(heads, kv, d, nq, nk):
    """Items that begin and end inside a token's heads."""
    print("causal wide groups", heads, kv, d, flush=True)
    _check(nq, nk, heads, kv, d, seed=17)
