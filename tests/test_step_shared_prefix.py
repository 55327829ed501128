"""Where tree positions start when the shared prefix of a step comes and goes: on the CPU, with the stand-in for the
library's handle of test_step_cache_budget.py."""
import torch

from test_step_cache_budget import CFG, step  # noqa: F401  (the fixture)


def _base(s):
    s.tree()
    return s.out["pos"][:, 0].tolist()


def _prefix(P):
    return torch.zeros(CFG.Hkv, P, CFG.D)


def test_positions_without_a_prefix_any_more(step):  # noqa: F811
    step.set_inputs(Kp=_prefix(6), Vp=_prefix(6), prefix_len=torch.tensor([6, 2], dtype=torch.int32))
    assert _base(step) == [10, 11]
    step.set_inputs(Kp=None, Vp=None)
    assert _base(step) == [4, 9]
    assert step.inp["prefix_len"] is None
    # a prefix that comes back needs lengths of its own (the library refuses a prefix without any)
    step.set_inputs(Kp=_prefix(3), Vp=_prefix(3), prefix_len=torch.tensor([3, 0], dtype=torch.int32))
    assert _base(step) == [7, 9]


def test_lengths_alone_are_no_prefix(step):  # noqa: F811
    step.enable_cache_budget(8, sinks=1, recent=2, Lcap=24)
    step.set_inputs(prefix_len=torch.tensor([6, 2], dtype=torch.int32))
    assert _base(step) == [4, 9]


def test_an_empty_prefix_is_no_prefix(step):  # noqa: F811
    step.set_inputs(Kp=_prefix(0), Vp=_prefix(0), prefix_len=torch.tensor([6, 2], dtype=torch.int32))
    assert _base(step) == [4, 9]


def test_the_attention_goes_back_to_its_own_form(step):  # noqa: F811
    """Without a prefix and without a budget a step makes the calls of one that never had a prefix: the shared form is
    slower there."""
    def made():
        step.h.calls.clear()
        step.tree()
        step.attention()
        return step.h.calls[1:]
    step.set_inputs(Q=None)
    assert made() == ["tree_attention"]
    step.set_inputs(Kp=_prefix(6), Vp=_prefix(6), prefix_len=torch.tensor([6, 2], dtype=torch.int32))
    assert made() == ["tree_attention_shared"]
    step.set_inputs(Kp=None)
    assert made() == ["tree_attention"] and _base(step) == [4, 9]
    step.enable_cache_budget(8, sinks=1, recent=2)
    assert made() == ["tree_attention_shared"]
