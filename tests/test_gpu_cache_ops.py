"""GPU parity of the cache operators (gathered attention weight, eviction) against the oracle.

Tolerance of the weights: a score is a float32 sum of D products (exact for bfloat16 inputs), off by at most
D 2^-24 sum|q k| scale; with N(0,1) inputs and scale 1/sqrt(D), sum|q k| scale is about 0.64 sqrt(D) and below
2 sqrt(D) in these tests, i.e. at most 128 * 2^-24 * 2 * 11.4 = 1.8e-4 absolute, which is the relative error of
its exponential; the sums of positive weights add (rows + log2) roundings of 2^-24.  RTOL 2e-4 covers both."""
import numpy as np
import pytest

from oracle import ctcsd_oracle as orc
from paper_2412_00061_b200 import binding

RTOL = 2e-4


def _handle(B, Hq, Hkv, D, dtype, T=5, max_nodes=16):
    return binding.Handle(B, 64, 50, T, 2, 8, 4, max_nodes, Hq, Hkv, D, binding.DTYPE_BF16 if dtype == "bf16" else binding.DTYPE_F32)


def _dev(a, act=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
    return t.to(act) if act is not None else t


def _host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _mass_inputs(rng, B, Hq, Hkv, D, dtype, T, max_nodes, kv_before, acc, Lcap):
    from paper_2412_00061_b200 import synth
    Q = synth.to_dtype(rng.normal(size=(B, max_nodes, Hq, D)).astype(np.float32), dtype)
    K = synth.to_dtype(rng.normal(size=(B, Hkv, Lcap, D)).astype(np.float32), dtype)
    acc = np.asarray(acc, dtype=np.int32)
    kv = (np.asarray(kv_before) + 1 + acc).astype(np.int32)
    path = np.full((B, T), -1, dtype=np.int32)
    lse = np.full((B, max_nodes, Hq), np.nan, dtype=np.float32)        # nodes off the path are never looked at
    scale = 1.0 / np.sqrt(D)
    grp = Hq // Hkv
    for b in range(B):
        path[b, :acc[b]] = np.sort(rng.choice(np.arange(1, max_nodes), size=acc[b], replace=False))
        for l, node in enumerate([0] + list(path[b, :acc[b]])):
            s = np.einsum("hd,hjd->hj", Q[b, node].astype(np.float64), np.repeat(K[b, :, :kv[b] - acc[b] + l], grp, axis=0)) * scale
            lse[b, node] = (np.log(np.exp(s).sum(-1)) + 0.3).astype(np.float32)
        off = [i for i in range(max_nodes) if i not in [0] + list(path[b, :acc[b]])]
        Q[b, off] = np.nan
        K[b, :, kv[b]:] = np.nan
    mass = rng.random((B, Hkv, Lcap)).astype(np.float32)
    pos = rng.integers(0, 999, (B, Hkv, Lcap)).astype(np.int32)
    return Q, K, kv, acc, path, lse, scale, mass, pos


MASS = {   # B, Hq, Hkv, D, T, max_nodes, cached rows before the step, accepted
    "one_row": (1, 4, 4, 64, 1, 4, [0], [0]),
    "token": (3, 8, 8, 128, 4, 2, [0, 127, 128], [0, 0, 1]),
    "borders": (4, 6, 3, 64, 5, 16, [123, 124, 125, 255], [5, 3, 2, 0]),
    "gqa": (5, 16, 2, 128, 6, 24, [700, 1, 0, 333, 64], [6, 6, 0, 2, 1]),
    "odd_group": (2, 15, 3, 64, 8, 9, [1000, 77], [8, 7]),
    "rows_past_one_pass": (2, 80, 2, 64, 8, 12, [300, 130], [8, 6]),       # 360 query rows per kv head
    "mqa": (2, 32, 1, 128, 3, 8, [515, 2], [3, 0]),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", sorted(MASS))
def test_gathered_weight(name, dtype):
    import torch
    B, Hq, Hkv, D, T, max_nodes, before, acc = MASS[name]
    rng = np.random.default_rng([5, sorted(MASS).index(name)])
    Lcap = max(before) + T + 1 + 7
    Q, K, kv, acc, path, lse, scale, mass, pos = _mass_inputs(rng, B, Hq, Hkv, D, dtype, T, max_nodes, before, acc, Lcap)
    lse[B - 1, 0, 0] = -np.inf                                             # a query that saw nothing adds nothing
    ev = rng.integers(0, 50, B).astype(np.int32)
    want_m, want_p = orc.attention_mass(Q, K, kv, acc, path, lse, scale, 0.75, mass, pos, ev)
    act = torch.bfloat16 if dtype == "bf16" else torch.float32
    h = _handle(B, Hq, Hkv, D, dtype, T, max_nodes)
    m, p = _dev(mass), _dev(pos)
    h.attention_mass(_dev(Q, act), _dev(K, act), _dev(kv), _dev(acc), _dev(path), _dev(lse), scale, m, p, _dev(ev), decay=0.75)
    assert h.poll_status() == 0
    got = _host(m)
    np.testing.assert_allclose(got, want_m, rtol=RTOL, atol=1e-12)
    np.testing.assert_array_equal(_host(p), want_p)
    for b in range(B):
        assert np.array_equal(got[b, :, kv[b]:], mass[b, :, kv[b]:])       # rows past the end stay as they were


@pytest.mark.gpu
def test_a_sequence_outside_its_arrays_is_reported_and_left_alone():
    import torch
    B, Hq, Hkv, D, T, nodes = 5, 4, 2, 64, 3, 8
    rng = np.random.default_rng(6)
    Q, K, kv, acc, path, lse, scale, mass, pos = _mass_inputs(rng, B, Hq, Hkv, D, "bf16", T, nodes, [40] * B, [2] * B, 60)
    good = 4
    kv2, acc2, path2 = kv.copy(), acc.copy(), path.copy()
    kv2[0] = 61                        # past the cache
    acc2[1] = 4                        # longer than T
    path2[2, 0] = 8                    # no such node
    kv2[3] = 2                         # shorter than the accepted path
    h = _handle(B, Hq, Hkv, D, "bf16", T, nodes)
    m, p = _dev(mass), _dev(pos)
    bf = torch.bfloat16
    h.attention_mass(_dev(Q, bf), _dev(K, bf), _dev(kv2), _dev(acc2), _dev(path2), _dev(lse), scale, m, p)
    assert h.poll_status() == -1 and h.poll_status() == 0
    want_m, want_p = orc.attention_mass(Q[good:], K[good:], kv[good:], acc[good:], path[good:], lse[good:], scale, 1.0,
                                        mass[good:], pos[good:])
    np.testing.assert_allclose(_host(m)[good:], want_m, rtol=RTOL, atol=1e-12)
    np.testing.assert_array_equal(_host(p)[good:], want_p)
    assert np.array_equal(_host(m)[:good], mass[:good]) and np.array_equal(_host(p)[:good], pos[:good])


def _evict_inputs(rng, B, Hkv, D, dtype, kv, Lcap, ties):
    from paper_2412_00061_b200 import synth
    K = synth.to_dtype(rng.normal(size=(B, Hkv, Lcap, D)).astype(np.float32), dtype)
    V = synth.to_dtype(rng.normal(size=(B, Hkv, Lcap, D)).astype(np.float32), dtype)
    mass = (rng.random((B, Hkv, Lcap)) ** 6).astype(np.float32)
    if ties:
        mass = np.round(mass * 4).astype(np.float32) / 4
        mass[rng.random(mass.shape) < 0.1] = -0.0
    ev = rng.integers(0, 300, B).astype(np.int32)
    pos = np.stack([np.stack([rng.permutation(Lcap) for _ in range(Hkv)]) for _ in range(B)]).astype(np.int32)
    return K, V, mass, pos, np.asarray(kv, dtype=np.int32), ev


EVICT = {   # B, Hkv, D, kv_len, Lcap, budget, sinks, recent
    "nothing_to_do": (3, 2, 64, [0, 5, 8], 16, 8, 1, 2),
    "to_one_row": (2, 3, 64, [1, 40], 40, 1, 0, 0),
    "one_row_leaves": (3, 4, 128, [65, 64, 66], 70, 64, 4, 16),
    "all_protected": (2, 2, 64, [33, 50], 50, 20, 10, 10),
    "ragged": (4, 3, 64, [700, 200, 0, 131], 701, 130, 3, 40),
    "cluster": (1, 2, 64, [5000], 5003, 1200, 4, 100),
    "half": (1, 8, 64, [8192], 8192, 4096, 0, 0),
}


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("name", sorted(EVICT))
def test_eviction(name, ties, dtype, in_place):
    import torch
    B, Hkv, D, kv, Lcap, budget, sinks, recent = EVICT[name]
    rng = np.random.default_rng([7, sorted(EVICT).index(name), int(ties)])
    K, V, mass, pos, kv, ev = _evict_inputs(rng, B, Hkv, D, dtype, kv, Lcap, ties)
    if ties:
        mass[:, :, 1::7] = np.nan
    for b in range(B):
        K[b, :, kv[b]:], V[b, :, kv[b]:], mass[b, :, kv[b]:] = np.nan, np.nan, 99.0     # never looked at
    want = orc.evict_rows(K, V, mass, pos, kv, ev, budget, sinks, recent)
    act = torch.bfloat16 if dtype == "bf16" else torch.float32
    h = _handle(B, Hkv, Hkv, D, dtype)
    plan = h.make_eviction(Lcap)
    Kd, Vd, md, pd, kd, ed = _dev(K, act), _dev(V, act), _dev(mass), _dev(pos), _dev(kv), _dev(ev)
    outs = (md, pd, kd, ed) if in_place else (torch.full_like(md, -3.0), torch.full_like(pd, -3), torch.zeros_like(kd), torch.zeros_like(ed))
    h.evict_rows(plan, Kd, Vd, md, pd, kd, ed, budget, sinks, recent, *outs)
    assert h.poll_status() == 0
    np.testing.assert_array_equal(_host(outs[2]), want[4])
    np.testing.assert_array_equal(_host(outs[3]), want[5])
    for b in range(B):
        n = int(want[4][b])
        for got, w in zip([Kd, Vd, outs[0], outs[1]], want[:4]):
            np.testing.assert_array_equal(_host(got)[b, :, :n], w[b, :, :n])
        if not in_place:
            assert np.all(_host(outs[1])[b, :, n:] == -3)                  # rows behind the new length are not written


@pytest.mark.gpu
def test_eviction_of_a_share_that_does_not_fit_in_shared_memory():
    """More rows per CTA than it keeps keys of (a cluster of one because there are many heads)."""
    import torch
    B, Hkv, D, L, budget = 2, 160, 64, 9000, 8900
    rng = np.random.default_rng(11)
    kv = np.array([L, 8500], dtype=np.int32)
    mass = np.round(rng.random((B, Hkv, L)) * 50).astype(np.float32)
    pos = np.tile(np.arange(L, dtype=np.int32), (B, Hkv, 1))
    ev = np.zeros(B, dtype=np.int32)
    K = torch.randn(B, Hkv, L, D, device="cuda:0").to(torch.bfloat16)
    V = torch.randn(B, Hkv, L, D, device="cuda:0").to(torch.bfloat16)
    K0 = K.clone()
    h = _handle(B, Hkv, Hkv, D, "bf16")
    md, pd, kd, ed = _dev(mass), _dev(pos), _dev(kv), _dev(ev)
    h.evict_rows(h.make_eviction(L), K, V, md, pd, kd, ed, budget, 4, 50, md, pd, kd, ed)
    assert h.poll_status() == 0
    assert kd.tolist() == [budget, 8500] and ed.tolist() == [100, 0]
    got = pd[0].cpu().numpy()
    for g in range(0, Hkv, 13):
        safe = (np.arange(L) < 4) | (np.arange(L) >= L - 50)
        kept = np.zeros(L, dtype=bool)
        kept[np.lexsort((np.arange(L), -mass[0, g], ~safe))[:budget]] = True
        src = np.arange(budget)
        src[~kept[:budget]] = budget + np.nonzero(kept[budget:])[0]
        np.testing.assert_array_equal(got[g, :budget], src)
        assert torch.equal(K[0, g, :budget], K0[0, g][torch.from_numpy(src).to("cuda:0")])
    assert torch.equal(K[1], K0[1])


@pytest.mark.gpu
def test_eviction_refuses_and_reports():
    import torch
    B, Hkv, D, Lcap = 2, 2, 64, 32
    h = _handle(B, Hkv, Hkv, D, "bf16")
    plan = h.make_eviction(Lcap)
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda:0")
    K, V = z(B, Hkv, Lcap, D), z(B, Hkv, Lcap, D)
    m, p = z(B, Hkv, Lcap, dtype=torch.float32), z(B, Hkv, Lcap, dtype=torch.int32)
    kv, ev = torch.full((B,), 20, dtype=torch.int32, device="cuda:0"), z(B, dtype=torch.int32)
    m2 = torch.zeros_like(m)
    for budget, sinks, recent in ((0, 0, 0), (8, -1, 0), (8, 0, -1), (8, 5, 4)):
        with pytest.raises(binding.CtcsdError):
            h.evict_rows(plan, K, V, m, p, kv, ev, budget, sinks, recent, m, p, kv, ev)
    with pytest.raises(binding.CtcsdError):
        h.evict_rows(plan, K, V, m, p, kv, ev, 8, 0, 0, m2, p, kv, ev)         # one array in place, the other not
    with pytest.raises(binding.CtcsdError):
        h.evict_rows(dict(plan, ws_bytes=plan["ws_bytes"] - 1), K, V, m, p, kv, ev, 8, 0, 0, m, p, kv, ev)
    kv2 = torch.tensor([33, 20], dtype=torch.int32, device="cuda:0")
    h.evict_rows(plan, K, V, m, p, kv2, ev, 8, 0, 0, m, p, kv2, ev)
    assert h.poll_status() == -1
    assert kv2.tolist() == [33, 8] and ev.tolist() == [0, 12]


def test_host_side_refusals_without_a_device():
    import ctypes
    lib = binding.load_library()
    n = ctypes.c_size_t(0)
    cfg = binding.CConfig(2, 64, 50, 5, 2, 8, 4, 16, 4, 2, 64, 1, 0, 0)
    assert lib.ctcsd_evict_rows_workspace_bytes(ctypes.byref(cfg), 100, ctypes.byref(n)) == 0 and n.value >= 4 * 2 * 2 * 100
    assert lib.ctcsd_evict_rows_workspace_bytes(ctypes.byref(cfg), 0, ctypes.byref(n)) == -1
    assert lib.ctcsd_evict_rows_workspace_bytes(None, 100, ctypes.byref(n)) == -1
    assert lib.ctcsd_attention_mass(*([None] * 4), 10, *([None] * 4), 1.0, 1.0, *([None] * 3)) == -1
    assert lib.ctcsd_evict_rows(None, None, None, 0, None, None, 10, *([None] * 4), 1, 0, 0, *([None] * 4)) == -1
