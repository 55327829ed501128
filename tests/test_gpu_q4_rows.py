"""Storing, appending and reading back rows of a 4-bit cache, bit for bit against the oracle.

Scale, origin and level are defined by float32 steps that both sides take, and a value is rounded once: nothing is off."""
import numpy as np
import pytest
import torch

import q4_util as u

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 1, 1, 64), ("bf16", 3, 7, 64), ("bf16", 2, 3, 128), ("fp32", 2, 3, 64), ("fp32", 1, 2, 128)]


def _rows(rng, B, Hkv, L, D, dtype):
    v = rng.normal(size=(B, Hkv, L, D)) * 10.0 ** rng.integers(-3, 3, (B, Hkv, L, 1)) + rng.normal(size=D)
    return torch.from_numpy(v.astype(np.float32)).to(u.DEV, u.act_of(dtype))


@pytest.mark.parametrize("dtype,B,Hkv,D", SHAPES)
@pytest.mark.parametrize("L", [1, 2, 33, 300])
def test_store_then_load(dtype, B, Hkv, D, L):
    rng = np.random.default_rng([L, D, B])
    h = u.handle(dtype, B=B, Hq=Hkv, Hkv=Hkv, D=D)
    cache = h.make_q4_cache(L + 9)
    for t in cache.values():
        t.view(torch.uint8).fill_(0x5a)
    K, V = _rows(rng, B, Hkv, L, D, dtype), _rows(rng, B, Hkv, L, D, dtype)
    n = rng.integers(0, L + 1, B)
    n[-1] = L
    at = rng.integers(0, 10, B)
    h.store_rows_q4(cache, K, V, u.i32(n), u.i32(at))
    out = torch.full_like(K, 7.0), torch.full_like(V, 7.0)
    h.load_rows_q4(cache, u.i32(at), u.i32(n), *out)
    assert h.poll_status() == 0
    for name, src, got in (("K", K, out[0]), ("V", V, out[1])):
        want = u.stands_for(src, 32, dtype)
        q, s, o = u.orc.q4_quantize(src.float().cpu().numpy(), 32)
        levels = u.levels_of(cache[name + "q"], D)
        pairs = cache[name + "s"].float().cpu().numpy()
        for b in range(B):
            assert torch.equal(got[b, :, :n[b]].double().cpu(), want[b, :, :n[b]])
            assert torch.count_nonzero(got[b, :, n[b]:]) == 0
            rows = slice(at[b], at[b] + n[b])
            np.testing.assert_array_equal(levels[b, :, rows], q[b, :, :n[b]])
            np.testing.assert_array_equal(pairs[b, :, rows, :, 0], s[b, :, :n[b]])
            np.testing.assert_array_equal(pairs[b, :, rows, :, 1], o[b, :, :n[b]])
            raw = cache[name + "q"][b].cpu().numpy()                 # other rows are left as they were
            assert np.all(raw[:, :at[b]] == 0x5a) and np.all(raw[:, at[b] + n[b]:] == 0x5a)
            raw = cache[name + "s"].view(torch.uint8)[b].cpu().numpy()
            assert np.all(raw[:, :at[b]] == 0x5a) and np.all(raw[:, at[b] + n[b]:] == 0x5a)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_groups_that_are_constant_or_hold_no_number(dtype):
    h = u.handle(dtype, D=128)
    K = torch.zeros(1, 1, 6, 128, device=u.DEV)
    K[0, 0, 1] = -3.25
    K[0, 0, 2, 5] = float("nan")
    K[0, 0, 3, 40] = float("inf")
    K[0, 0, 4, 70], K[0, 0, 4, 71] = 3e38, -3e38          # the range leaves float32
    K[0, 0, 5, 3] = -float("inf")
    K = K.to(u.act_of(dtype))
    cache = h.make_q4_cache(6)
    h.store_rows_q4(cache, K, -K, u.i32([6]))
    out = torch.empty_like(K), torch.empty_like(K)
    h.load_rows_q4(cache, None, u.i32([6]), *out)
    for got, src in ((out[0], K), (out[1], -K)):
        np.testing.assert_array_equal(got.double().cpu().numpy(), u.stands_for(src, 32, dtype).numpy())
    assert torch.isnan(out[0][0, 0, 4, 64:96]).all() and torch.equal(out[0][0, 0, 1], K[0, 0, 1])


@pytest.mark.parametrize("dtype,B,Hkv,D", SHAPES)
@pytest.mark.parametrize("in_place", [False, True])
def test_commit(dtype, B, Hkv, D, in_place):
    nodes, T = 9, 5
    rng = np.random.default_rng([B, D])
    h = u.handle(dtype, B=B, T=T, nodes=nodes, Hq=Hkv, Hkv=Hkv, D=D)
    kv = rng.integers(0, 30, B)
    acc = rng.integers(0, T + 1, B)
    acc[0], acc[-1] = (0, T) if B > 1 else (T, T)
    Lcap = int((kv + 1 + acc).max())                       # the longest sequence just fits
    path = np.full((B, T), -1)
    for b in range(B):
        path[b, :acc[b]] = np.sort(rng.choice(np.arange(1, nodes), acc[b], replace=False))
    Kt, Vt = _rows(rng, B, Hkv, nodes, D, dtype), _rows(rng, B, Hkv, nodes, D, dtype)
    cache = h.make_q4_cache(Lcap)
    for t in cache.values():
        t.view(torch.uint8).fill_(0x33)
    kv_len = u.i32(kv)
    new_len = kv_len if in_place else u.i32([0] * B)
    sel = u.i32([0] * B)
    h.commit_accepted_q4(Kt, Vt, cache, kv_len, u.i32(acc), u.i32(path), new_len, sel)
    out = torch.empty(B, Hkv, T + 1, D, dtype=Kt.dtype, device=u.DEV), torch.empty(B, Hkv, T + 1, D, dtype=Kt.dtype, device=u.DEV)
    h.load_rows_q4(cache, u.i32(kv), u.i32(acc + 1), *out)
    assert h.poll_status() == 0
    np.testing.assert_array_equal(new_len.cpu().numpy(), kv + 1 + acc)
    for b in range(B):
        at = [0] + list(path[b, :acc[b]])
        assert int(sel[b]) == b * nodes + at[-1]
        for src, got, name in ((Kt, out[0], "Kq"), (Vt, out[1], "Vq")):
            assert torch.equal(got[b, :, :acc[b] + 1].double().cpu(), u.stands_for(src, 32, dtype)[b][:, at])
            raw = cache[name][b].cpu().numpy()
            assert np.all(raw[:, :kv[b]] == 0x33) and np.all(raw[:, kv[b] + 1 + acc[b]:] == 0x33)


def test_sequences_that_leave_their_arrays_are_left_unchanged():
    B, nodes, T, D, L = 8, 6, 4, 64, 10
    h = u.handle("bf16", B=B, T=T, nodes=nodes, D=D)
    K = torch.randn(B, 1, L, D, device=u.DEV).to(torch.bfloat16)
    cache = h.make_q4_cache(L)
    fresh = {k: t.clone() for k, t in cache.items()}
    h.store_rows_q4(cache, K, K, u.i32([3, -1, L + 1, L, 2, 0, 5, 1]), u.i32([0, 0, 0, 1, -1, L, L - 5, L]))
    assert h.poll_status() == -1
    for b, fits in enumerate([True, False, False, False, False, False, True, False]):
        assert torch.equal(cache["Kq"][b], fresh["Kq"][b]) != fits
    out = torch.full((B, 1, 4, D), 5.0, dtype=torch.bfloat16, device=u.DEV), torch.full((B, 1, 4, D), 5.0, dtype=torch.bfloat16, device=u.DEV)
    h.load_rows_q4(cache, u.i32([0, 0, L - 3, 0, -1, 0, L - 5, L]), u.i32([3, 5, 4, -1, 2, 0, 4, 0]), *out)
    assert h.poll_status() == -1
    for b, fits in enumerate([True, False, False, False, False, False, True, False]):
        assert (torch.count_nonzero(out[0][b]) > 0) == fits
    before = {k: t.clone() for k, t in cache.items()}
    Kt = torch.randn(B, 1, nodes, D, device=u.DEV).to(torch.bfloat16)
    path = [[1, 2, -1, -1], [0, 2, -1, -1], [1, nodes, -1, -1], [-1] * 4, [1, 2, 3, 4], [-1] * 4, [1, 2, 3, 4], [2, 3, -1, -1]]
    new_len, sel = u.i32([0] * B), u.i32([0] * B)
    h.commit_accepted_q4(Kt, Kt, cache, u.i32([3, 3, 3, -1, 3, 3, L - 4, 3]), u.i32([2, 2, 2, 0, 5, -1, 4, 2]), u.i32(path), new_len, sel)
    assert h.poll_status() == -1
    for b, fits in enumerate([True, False, False, False, False, False, False, True]):
        assert torch.equal(cache["Kq"][b], before["Kq"][b]) != fits
    assert new_len.tolist() == [6, 3, 3, -1, 3, 3, L - 4, 6]
    assert sel.tolist() == [2] + [b * nodes for b in range(1, 7)] + [7 * nodes + 3]


def test_rows_behind_2_to_the_32_bytes():
    """One cache of 4.9 GB of levels for K: rows of its last head."""
    D, Lcap = 128, 4_800_000
    h = u.handle("bf16", B=1, Hq=16, Hkv=16, D=D)
    Q = torch.empty(1, 16, Lcap, D // 2, dtype=torch.uint8, device=u.DEV)
    S = torch.empty(1, 16, Lcap, D // 32, 2, dtype=torch.bfloat16, device=u.DEV)
    cache = dict(Kq=Q, Ks=S, Vq=torch.empty_like(Q), Vs=torch.empty_like(S))
    K = torch.randn(1, 16, 5, D, device=u.DEV).to(torch.bfloat16)
    V = torch.randn(1, 16, 5, D, device=u.DEV).to(torch.bfloat16)
    at = u.i32([Lcap - 5])
    h.store_rows_q4(cache, K, V, u.i32([5]), at)
    out = torch.empty_like(K), torch.empty_like(K)
    h.load_rows_q4(cache, at, u.i32([5]), *out)
    assert h.poll_status() == 0
    assert torch.equal(out[0].double().cpu(), u.stands_for(K, 32, "bf16")) and torch.equal(out[1].double().cpu(), u.stands_for(V, 32, "bf16"))
