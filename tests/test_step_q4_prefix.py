"""A 4-bit cache beside a prefix without rows: on the CPU, with the stand-in of test_step_q4.py."""
import pytest
import torch

from test_step_cache_budget import CFG, LCAP, step  # noqa: F401  (the fixtures)
from test_step_q4 import _calls, q4_step  # noqa: F401


def _prefix(rows):
    return dict(Kp=torch.zeros(CFG.Hkv, rows, CFG.D), Vp=torch.zeros(CFG.Hkv, rows, CFG.D), prefix_len=torch.zeros(CFG.B, dtype=torch.int32))


def test_a_prefix_without_rows_is_none(q4_step):  # noqa: F811
    s = q4_step
    s.set_inputs(**_prefix(0))
    s.use_q4_cache(LCAP)                       # nothing of a prefix is there
    s.set_inputs(**_prefix(0))
    assert _calls(s, "attention", "commit") == ["tree_attention_q4", "commit_accepted_q4"]
    with pytest.raises(ValueError):
        s.set_inputs(**_prefix(3))
    assert s.inp["Kp"].shape[1] == 0
    assert s._tree_base() is s.inp["kv_len"]
