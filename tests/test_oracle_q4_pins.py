"""Pins of the oracle's 4-bit format against facts that do not depend on how it is written."""
import numpy as np
import torch

from oracle import ctcsd_oracle as orc


def test_rounding_to_bfloat16_is_torchs():
    rng = np.random.default_rng(3)
    a = np.concatenate([rng.normal(size=4000) * 10.0 ** rng.integers(-6, 7, 4000), [0.0, 1.00390625, 1.01171875, -2.5]])
    a = a.astype(np.float32)
    want = torch.from_numpy(a).to(torch.bfloat16).double().numpy()
    np.testing.assert_array_equal(orc.round_to_bf16(a), want)


def test_values_lie_within_half_a_level_of_what_was_stored():
    """A level is off by half a scale at most; the scale's rounding (2^-8) can leave the largest value 31 scales of
    that short (level 15 stands 31 scales from the origin), and the origin's is 2^-8 of it."""
    rng = np.random.default_rng(4)
    v = (rng.normal(size=(50, 96)) * 10.0 ** rng.integers(-3, 3, (50, 1)) + rng.normal(size=(50, 1))).astype(np.float32)
    for group in (32, 64):
        q, s, o = orc.q4_quantize(v, group)
        assert q.min() >= 0 and q.max() <= 15
        back = orc.q4_values(q, s, o, group, False)
        at = np.arange(96) // group
        bound = 0.5 * s[..., at] + 31 * s[..., at] * 2.0 ** -8 + np.abs(o[..., at]) * 2.0 ** -8 + np.abs(back) * 2.0 ** -23
        assert np.all(np.abs(back - v) <= bound)


def test_constant_groups_zeros_and_groups_without_a_value():
    v = np.zeros((4, 64), dtype=np.float32)
    v[1] = 2.5
    v[2, 40] = np.nan
    v[3, 3] = np.inf
    q, s, o = orc.q4_quantize(v, 32)
    back = orc.q4_values(q, s, o, 32, True)
    np.testing.assert_array_equal(back[0], 0.0)
    np.testing.assert_array_equal(back[1], 2.5)
    assert np.all(np.isnan(back[2, 32:])) and np.all(back[2, :32] == 0)
    assert np.all(np.isnan(back[3, :32])) and np.all(back[3, 32:] == 0)
    assert np.all(q == 0)


def test_levels_that_are_values_come_back_as_themselves():
    """Sixteen evenly spaced values that a level can stand for exactly are kept; a short last group is a group of its own."""
    v = np.concatenate([np.tile(np.arange(16, dtype=np.float32) * 0.25 - 1.0, 2), [8.0, 23.0, 9.0, 10.0]])[None].astype(np.float32)
    q, s, o = orc.q4_quantize(v, 32)
    np.testing.assert_array_equal(orc.q4_values(q, s, o, 32, True), v)
    np.testing.assert_array_equal(q[0], list(range(16)) * 2 + [0, 15, 1, 2])
