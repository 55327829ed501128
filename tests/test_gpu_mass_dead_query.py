"""Attention mass: a query whose log-sum-exp is -inf adds nothing, whatever its row of Q holds.  (The shared-prefix attention
writes -inf for unused nodes, a finished sequence's root among them, and looks at none of their queries.)"""
import pytest

from test_gpu_mass_blocks import _call, _compare, _inputs

pytestmark = pytest.mark.gpu

CASES = {   # dtype, Hq, T
    "one_tile": ("bf16", 4, 5), "two_tiles": ("bf16", 8, 3), "tensor_memory": ("bf16", 64, 4), "two_passes": ("bf16", 128, 8),
    "fp32": ("fp32", 8, 5), "fp32_two_chunks": ("fp32", 64, 8),
}


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", sorted(CASES))
def test_a_query_that_saw_nothing_adds_nothing(name, bad):
    dtype, Hq, T = CASES[name]
    x = _inputs(3, Hq, 2, 128, dtype, T, 12, 0, 700, seed=40 + sorted(CASES).index(name))
    neg = -float("inf")
    # a finished sequence: nothing but an unused root
    x["kv"][1] -= x["acc"][1]
    x["acc"][1] = 0
    x["lse"][1], x["Q"][1] = neg, bad
    # an accepted node, and one head of the root
    node = int(x["path"][0, x["acc"][0] - 1])
    x["lse"][0, node], x["Q"][0, node] = neg, bad
    x["lse"][0, 0, Hq // 2], x["Q"][0, 0, Hq // 2] = neg, bad
    want_Q = x["Q"].clone()
    got = _call(x, dtype, 0.75)
    x["Q"] = want_Q.nan_to_num(0.0, 0.0, 0.0)            # (the restatement leaves them out by their log-sum-exp)
    _compare(x, got, 0.75)
    assert bool((got[0][1, :, int(x["kv"][1]) - 1] == 0).all())
