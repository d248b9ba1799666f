"""Linear attention with a decay per head: what its documentation says of starts from zeros, of values that are not finite, of cuts."""
import pytest
import torch

import linattn_testlib as T
from linattn_testlib import Problem
from serving_testlib import same_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,lens", [(2, [130, 0, 64, 1]), (1, [2300, 0, 700])])
def test_without_initial_states_every_sequence_started_from_zeros(H, lens, dtype):
    """No pool to resume from: the flags that say `resume` have nothing to resume, and the gradient of a start from zeros is zeros."""
    slots = list(range(len(lens)))[::-1]
    asks = Problem(lens, H, 1, 64, 64, dtype, seed=2, tail=3, resume=[1] * len(lens), slots=slots, backward=True)
    fresh = Problem(lens, H, 1, 64, 64, dtype, seed=2, tail=3, resume=[0] * len(lens), slots=slots, backward=True)
    for a, b in zip(asks.run(s_in=None), fresh.run()):
        assert same_bits(a, b)
    *grads, ds = asks.run_backward(s_in=None)
    *want, ds_want = fresh.run_backward()
    for a, b in zip(grads, want):
        assert same_bits(a, b)
    for s in slots:
        assert (ds[s] == 0).all() and (ds_want[s] == 0).all()
