"""A 4-bit cache and packed weights begun again: what DraftVerifyStep keeps, because captured graphs use it, on the CPU with the stand-in for
the library's handle of test_step_cache_budget.py."""
import pytest
import torch

from test_step_cache_budget import CFG, LCAP, step  # noqa: F401  (the fixture)


@pytest.fixture()
def q4_step(step):  # noqa: F811
    def quantize(Wd, group, stream=None, out=None):
        out = dict(w=torch.zeros(4), group=group) if out is None else out
        out["w"].fill_(float(Wd))
        return out

    step.h.quantize_weights_q4 = quantize
    step.h.make_q4_cache = lambda Lcap: {k: torch.zeros(Lcap) for k in ("Kq", "Ks", "Vq", "Vs")}
    step.h.make_q4_attention = lambda: dict(ws=torch.zeros(1))
    step.set_inputs(x=torch.zeros(CFG.B, CFG.H), Q=None, Kt=None, Vt=None)
    return step


def _held(s):
    return list(s.q4["cache"].values()) + [s.q4["ws"]["ws"], s.out["attn_lse"]]


def test_an_empty_cache_of_the_same_size_stands_in_the_same_tensors(q4_step):
    s = q4_step
    cache = s.use_q4_cache(LCAP)
    held = _held(s)
    for t in cache.values():
        t.fill_(3.0)
    assert s.use_q4_cache(LCAP) is cache
    assert all(a is b for a, b in zip(_held(s), held))
    assert all(torch.count_nonzero(t) == 0 for t in cache.values())


def test_a_cache_of_another_size_takes_the_rest_along(q4_step):
    s = q4_step
    cache = s.use_q4_cache(LCAP)
    held = _held(s)
    assert s.use_q4_cache(LCAP + 1) is not cache and s.q4["cache"]["Kq"].numel() == LCAP + 1
    assert all(a is b for a, b in zip(_held(s)[4:], held[4:]))
    with pytest.raises(ValueError):
        s.use_q4_cache(0)
    assert s.q4["cache"]["Kq"].numel() == LCAP + 1


def test_the_log_sum_exp_stays_where_it_is_when_other_attention_joins(q4_step):
    s = q4_step
    s.use_q4_cache(LCAP)
    lse = s.out["attn_lse"]
    s._use_shared_attention()
    assert s.out["attn_lse"] is lse
    s.use_q4_cache(LCAP)
    assert s.out["attn_lse"] is lse


def test_weights_packed_again_stand_where_they_stood(q4_step):
    s = q4_step
    W = torch.ones(1)
    s.set_inputs(Wd=W)
    packed = s.quantize_draft_weights(64)
    w = packed["w"]
    W.fill_(2.0)                                # the same weights, trained further
    assert s.quantize_draft_weights(64) is packed and s.inp["Wd_q4"] is packed and packed["w"] is w and torch.all(w == 2.0)
    assert s.quantize_draft_weights(32) is not packed and torch.all(w == 2.0)         # another group: another layout
    # other weights: packed ones that the caller holds are left alone
    first = s.inp["Wd_q4"]
    s.set_inputs(Wd=torch.full((1,), 5.0))
    assert s.quantize_draft_weights(32) is not first and torch.all(first["w"] == 2.0)
