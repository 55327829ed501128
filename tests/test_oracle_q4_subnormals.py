"""The oracle's rounding to bfloat16 where numbers are subnormal (spacing 2^-133), and what that makes of levels."""
import numpy as np
import torch

from oracle import ctcsd_oracle as orc


def test_rounding_to_subnormal_bfloat16_is_torchs():
    rng = np.random.default_rng(5)
    a = (rng.normal(size=6000) * np.ldexp(1.0, rng.integers(-149, -110, 6000))).astype(np.float32)
    steps = np.ldexp(np.arange(0, 600, dtype=np.float64) / 2, -133).astype(np.float32)       # every second one lies between two numbers
    a = np.concatenate([a, steps, -steps])
    want = torch.from_numpy(a).to(torch.bfloat16).double().numpy()
    np.testing.assert_array_equal(orc.round_to_bf16(a), want)


def test_levels_of_a_subnormal_scale_stay_within_0_and_15():
    """Limits whose scale has six significant bits: (v - origin) / scale - 16 is 15.9 at the largest value, which rounds to 16."""
    v = np.linspace(-3.2192902e-37, -2.6344046e-37, 32)[None].astype(np.float32)
    q, s, o = orc.q4_quantize(v, 32)
    assert 0 < s[0, 0] < 2.0 ** -126 and s[0, 0] == np.float64(torch.tensor(s[0, 0]).to(torch.bfloat16))
    exact = (v[0].astype(np.float64) - o[0, 0]) / s[0, 0] - 16.0
    assert exact.max() > 15.5 and q.max() == 15 and q.min() >= 0
