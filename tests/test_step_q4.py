"""Which calls a step makes with 4-bit weights and a 4-bit cache, and what it refuses: on the CPU, with the stand-in for the
library's handle of test_step_cache_budget.py."""
import pytest
import torch

from test_step_cache_budget import CFG, LCAP, _chain, step  # noqa: F401  (the fixture)


@pytest.fixture()
def q4_step(step):  # noqa: F811
    """The stand-in with the 4-bit calls that return something."""
    step.h.quantize_weights_q4 = lambda Wd, group, stream=None: dict(w=Wd, group=group)
    step.h.make_q4_cache = lambda Lcap: dict(Lcap=Lcap)
    step.h.make_q4_attention = lambda: dict(ws=None)
    step.set_inputs(x=torch.zeros(CFG.B, CFG.H), Q=None, Kt=None, Vt=None)
    return step


def _calls(s, *stages):
    s.h.calls.clear()
    for stage in stages:
        getattr(s, stage)()
    return list(s.h.calls)


def test_weights_in_4_bits_until_others_are_given(q4_step):
    s = q4_step
    with pytest.raises(ValueError):
        s.quantize_draft_weights()
    W = torch.zeros(1)
    s.set_inputs(Wd=W)
    assert _calls(s, "draft") == ["draft_logits"]
    assert s.quantize_draft_weights(64)["group"] == 64
    assert _calls(s, "draft") == ["draft_logits_q4"]
    s.set_inputs(Wd=None)                       # the 16-bit weights are let go
    assert _calls(s, "draft") == ["draft_logits_q4"]
    s.set_inputs(x=s.inp["x"])
    assert _calls(s, "draft") == ["draft_logits_q4"]
    s.set_inputs(Wd=W)                          # new weights: the packed ones are not theirs
    assert _calls(s, "draft") == ["draft_logits"]
    s.set_inputs(Wd=W, Wd_q4=dict(w=W, group=32))
    assert _calls(s, "draft") == ["draft_logits_q4"]


def test_a_4_bit_cache_takes_the_step_over(q4_step):
    s = q4_step
    with pytest.raises(ValueError):
        s.store_prompt(None, None, None)
    assert _calls(s, "attention", "commit") == ["tree_attention", "commit_accepted"]
    assert s.use_q4_cache(17) == dict(Lcap=17)
    assert _calls(s, "attention", "commit") == ["tree_attention_q4", "commit_accepted_q4"]
    s.store_prompt(None, None, None)
    assert s.h.calls[-1] == "store_rows_q4"
    assert s.use_q4_cache() == dict(Lcap=CFG.Lcap)
    with pytest.raises(ValueError):
        s.use_q4_cache(0)


def test_no_prefix_and_no_budget_beside_a_4_bit_cache(q4_step):
    s = q4_step
    prefix = dict(Kp=torch.zeros(CFG.Hkv, 3, CFG.D), Vp=torch.zeros(CFG.Hkv, 3, CFG.D), prefix_len=torch.zeros(CFG.B, dtype=torch.int32))
    s.use_q4_cache(LCAP)
    with pytest.raises(ValueError):
        s.set_inputs(**prefix)
    assert s.inp.get("Kp") is None
    with pytest.raises(ValueError):
        s.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    s.set_inputs(Kp=None)
    s.q4 = None
    s.set_inputs(**prefix)
    with pytest.raises(ValueError):
        s.use_q4_cache(LCAP)
    s.set_inputs(Kp=None)
    s.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    with pytest.raises(ValueError):
        s.use_q4_cache(LCAP)


def test_chained_steps_hand_their_tables_over_as_tree_rows(q4_step):
    s = q4_step
    s.set_inputs(Wd=torch.zeros(1))
    s.quantize_draft_weights()
    s.use_q4_cache(LCAP)
    _chain(s, 2)
    s.h.calls.clear()
    s.run_chain()
    made = [c for c in s.h.calls if "q4" in c]
    assert made == ["draft_logits_q4", "tree_attention_q4", "commit_accepted_q4"] * 2
    assert not any(c in ("draft_logits", "draft_logits_rows", "tree_attention", "commit_accepted") for c in s.h.calls)
    assert s.inp["Kt"].data_ptr() == s.chain["Ktab"][1].data_ptr()
