"""Life and arguments of causal plans on the host."""
import copy
import gc
import weakref

import numpy as np
import pytest

import paper_2606_13872_amd as sra


def test_a_copied_plan_outlives_the_first():
    plan = sra.CausalPlan([300, 40], 4, 2, 64)
    want = [plan.mask(which, b, 1) for which in range(3) for b in range(2)]
    held = weakref.ref(plan._handle)
    other = copy.copy(plan)
    del plan
    gc.collect()
    assert other._handle is held()  # still owned, so not destroyed
    made = [sra.CausalPlan([7 * i + 1], 4, 2, 64) for i in range(8)]  # would take the memory of a destroyed one
    got = [other.mask(which, b, 1) for which in range(3) for b in range(2)]
    assert all(np.array_equal(a, b) for a, b in zip(got, want)) and len(made) == 8
    del other
    gc.collect()
    assert held() is None


@pytest.mark.parametrize("sizes", [(2**32 + 8, 2, 64), (8, 2**32 + 2, 64), (8, 2, 2**32 + 64), (-2**32 + 8, 2, 64)])
def test_sizes_past_32_bits_are_refused(sizes):
    """They would reach the library cut to their lower 32 bits."""
    with pytest.raises(sra.SRAError) as e:
        sra.CausalPlan([3], *sizes)
    assert e.value.status == 1
