"""A step that goes back from a 4-bit cache to 16-bit rows: on the CPU, with the stand-in of test_step_q4.py."""
import pytest
import torch

from test_step_cache_budget import CFG, LCAP, step  # noqa: F401  (the fixtures)
from test_step_q4 import _calls, q4_step  # noqa: F401


def _prefix(rows):
    return dict(Kp=torch.zeros(CFG.Hkv, rows, CFG.D), Vp=torch.zeros(CFG.Hkv, rows, CFG.D), prefix_len=torch.zeros(CFG.B, dtype=torch.int32))


def test_a_step_goes_back_to_16_bit_rows(q4_step):  # noqa: F811
    s = q4_step
    with pytest.raises(ValueError):
        s.leave_q4_cache()
    s.use_q4_cache(LCAP)
    s.leave_q4_cache()
    assert s.q4 is None and _calls(s, "attention", "commit") == ["tree_attention", "commit_accepted"]
    with pytest.raises(ValueError):
        s.store_prompt(None, None, None)
    s.set_inputs(**_prefix(3))                 # what goes with 16-bit rows only is open again
    s.set_inputs(Kp=None)
    s.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    assert _calls(s, "attention") == ["tree_attention_shared"]
