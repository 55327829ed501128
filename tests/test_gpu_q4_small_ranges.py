"""Groups whose range is so small that their scale is a subnormal bfloat16 number (below 2^-126, with fewer significant bits), around
that border and far from it: levels, scales and origins bit for bit against the oracle, for cached rows and for packed weights.

Scale, origin and level are defined by float32 steps that both sides take, and a value is rounded once: nothing is off."""
import numpy as np
import pytest
import torch

import q4_util as u

pytestmark = pytest.mark.gpu


def small_rows(rows, n):
    """Rows whose groups of 32 have ranges of 2^-140 .. 2^-112, at offsets of up to 100 ranges (the first row: a pair of limits whose
    largest value stands 15.6 scales above the smallest, so that rounding alone leads past level 15)."""
    rng = np.random.default_rng([rows, n])
    span = np.ldexp(1.0, rng.integers(-140, -111, (rows, n // 32, 1))) * rng.uniform(0.5, 1.0, (rows, n // 32, 1))
    v = (rng.uniform(0.0, 1.0, (rows, n // 32, 32)) + np.where(rng.random((rows, n // 32, 1)) < 0.5, 0.0, rng.uniform(-100, 100, (rows, n // 32, 1)))) * span
    v[..., 0] = v.min(-1)
    v[0] = np.linspace(-3.2192902e-37, -2.6344046e-37, 32)
    return v.reshape(rows, n).astype(np.float32)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_cached_rows_of_small_ranges(dtype, D):
    L = 600
    h = u.handle(dtype, D=D)
    cache = h.make_q4_cache(L)
    K = torch.from_numpy(small_rows(L, D)).to(u.DEV, u.act_of(dtype)).reshape(1, 1, L, D)
    h.store_rows_q4(cache, K, -K, u.i32([L]))
    out = torch.empty_like(K), torch.empty_like(K)
    h.load_rows_q4(cache, None, u.i32([L]), *out)
    assert h.poll_status() == 0
    for name, src, got in (("K", K, out[0]), ("V", -K, out[1])):
        q, s, o = u.orc.q4_quantize(src.float().cpu().numpy(), 32)
        assert np.any((s > 0) & (s < 2.0 ** -126)) and np.any(s >= 2.0 ** -126)
        pairs = cache[name + "s"].float().cpu().numpy()
        np.testing.assert_array_equal(pairs[..., 0], s)
        np.testing.assert_array_equal(pairs[..., 1], o)
        np.testing.assert_array_equal(u.levels_of(cache[name + "q"], D), q)
        np.testing.assert_array_equal(got.double().cpu().numpy(), u.orc.q4_values(q, s, o, 32, dtype == "bf16"))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_packed_weights_of_small_ranges(dtype):
    H, V, group = 256, 63, 32
    h = u.handle(dtype, H=H, V=V, T=1, k=1)
    W = torch.from_numpy(small_rows(V + 1, H)).to(u.DEV, u.act_of(dtype)).reshape(1, V + 1, H)
    words = h.quantize_weights_q4(W, group)["w"].cpu().numpy().view("<u4").reshape(4, 2, (1024 + 256) // 4)
    q, s, o = u.orc.q4_quantize(W.float().cpu().numpy(), group)
    for v in range(V + 1):
        for h0 in range(0, H, 8):
            w = int(words[v // 16, h0 // 128, 64 * (h0 % 128 // 32) + 4 * (v % 16) + h0 % 32 // 8])
            assert [((w | w << 32) >> bit) & 15 for bit in u.WORD_BITS] == list(q[0, v, h0:h0 + 8])
            so = int(words[v // 16, h0 // 128, 256 + (v % 16) * 4 + h0 % 128 // 32])
            pair = [np.array([x], dtype="<u4").view("<f4")[0] for x in ((so & 0xffff) << 16, so & 0xffff0000)]
            assert pair == [s[0, v, h0 // 32], o[0, v, h0 // 32]]
