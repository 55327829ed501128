"""The cache operators at edges that test_gpu_cache_ops.py and test_gpu_cache_chain.py leave out: infinite weights in an eviction,
caches whose last head begins behind 2^32 elements, and chained steps that keep a budget without a shared prefix.
Tolerances as derived there: outputs 2e-2 (bf16) / 2e-4 (fp32), log-sum-exp 3e-4, weights 2e-4 relative; the rest exact."""
import math

import numpy as np
import pytest

from oracle import ctcsd_oracle as orc
from paper_2412_00061_b200 import binding, synth
from test_gpu_cache_chain import SHAPES, _chain
from test_gpu_cache_ops import EVICT, _dev, _evict_inputs, _handle, _host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("share", [0.02, 0.6])
@pytest.mark.parametrize("name", sorted(EVICT))
def test_infinite_weights(name, share, dtype):
    """+inf ranks above every finite weight, -inf below, NaN last; equal ones go by row."""
    import torch
    B, Hkv, D, kv, Lcap, budget, sinks, recent = EVICT[name]
    rng = np.random.default_rng([9, sorted(EVICT).index(name), int(share * 100)])
    K, V, mass, pos, kv, ev = _evict_inputs(rng, B, Hkv, D, dtype, kv, Lcap, False)
    u = rng.random(mass.shape)
    mass[u < share] = np.inf
    mass[(u >= share) & (u < share + 0.2)] = -np.inf
    mass[(u >= share + 0.2) & (u < share + 0.3)] = np.nan
    want = orc.evict_rows(K, V, mass, pos, kv, ev, budget, sinks, recent)
    act = torch.bfloat16 if dtype == "bf16" else torch.float32
    h = _handle(B, Hkv, Hkv, D, dtype)
    Kd, Vd, md, pd, kd, ed = _dev(K, act), _dev(V, act), _dev(mass), _dev(pos), _dev(kv), _dev(ev)
    h.evict_rows(h.make_eviction(Lcap), Kd, Vd, md, pd, kd, ed, budget, sinks, recent, md, pd, kd, ed)
    assert h.poll_status() == 0
    np.testing.assert_array_equal(_host(kd), want[4])
    for b in range(B):
        n = int(want[4][b])
        for got, w in zip([Kd, Vd, md, pd], want[:4]):
            np.testing.assert_array_equal(_host(got)[b, :, :n], w[b, :, :n])


def test_a_head_behind_32_bits():
    """Three sequences of two heads; the last sequence's heads begin past 2^32 elements and hold what the attention and the
    gathered weight read, the heads before them hold other rows."""
    import torch
    B, Hq, Hkv, D, nodes, T, kv, n = 3, 4, 2, 128, 8, 3, 300, 5
    Lcap = (1 << 30) // D + 4096
    rng = np.random.default_rng(71)
    h = binding.Handle(B, 64, 50, T, 2, 8, 4, nodes, Hq, Hkv, D, binding.DTYPE_BF16)
    dev, bf = "cuda:0", torch.bfloat16
    K = torch.zeros(B, Hkv, Lcap, D, dtype=bf, device=dev)
    V = torch.zeros_like(K)
    assert 4 * Lcap * D > 1 << 32                       # where the last sequence begins
    r = lambda *s: synth.to_dtype(rng.normal(size=s).astype(np.float32), "bf16")
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
    Ks, Vs, Q = r(B, Hkv, kv + n, D), r(B, Hkv, kv + n, D), r(B, nodes, Hq, D)
    K[:, :, :kv + n], V[:, :, :kv + n] = d(Ks).to(bf), d(Vs).to(bf)
    mask = np.zeros((B, nodes, 1), dtype=np.uint64)
    for i in range(n):
        mask[:, i, 0] = (1 << (i + 1)) - 1
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)
    O, lse = torch.zeros(B, nodes, Hq, D, dtype=bf, device=dev), torch.zeros(B, nodes, Hq, device=dev)
    scale = 1 / math.sqrt(D)
    h.tree_attention_shared(h.make_shared_attention(), d(Q).to(bf), None, None, None, K, V, i32(*[kv] * B), i32(*[n] * B),
                            d(mask.view(np.int64)), scale, O, lse)
    want_O, want_lse = orc.tree_attention_shared(Q, np.zeros((Hkv, 0, D)), np.zeros((Hkv, 0, D)), [0] * B, Ks, Vs, [kv] * B, [n] * B, mask, scale)
    assert h.poll_status() == 0
    assert np.max(np.abs(O.float().cpu().numpy() - want_O)) <= 2e-2 + 2.0 ** -8
    f = np.isfinite(want_lse)
    assert np.max(np.abs(lse.cpu().numpy()[f] - want_lse[f])) <= 3e-4
    mass = torch.zeros(B, Hkv, Lcap, device=dev)
    pos = torch.full((B, Hkv, Lcap), -1, dtype=torch.int32, device=dev)
    path = np.tile(np.array([1, 2, -1], dtype=np.int32), (B, 1))
    h.attention_mass(d(Q).to(bf), K, i32(*[kv + 3] * B), i32(*[2] * B), d(path), lse, scale, mass, pos)
    assert h.poll_status() == 0
    want_m, want_p = orc.attention_mass(Q, Ks, np.array([kv + 3] * B), np.array([2] * B), path, lse.cpu().numpy(), scale, 1.0,
                                        np.zeros((B, Hkv, kv + n)), np.full((B, Hkv, kv + n), -1))
    np.testing.assert_allclose(mass[:, :, :kv + n].cpu().numpy(), want_m, rtol=2e-4, atol=1e-9)
    np.testing.assert_array_equal(pos[:, :, :kv + n].cpu().numpy(), want_p)
    assert mass[:, :, kv + n:].abs().max().item() == 0


@pytest.mark.parametrize("name", sorted(SHAPES))
def test_a_budget_without_a_shared_prefix(name):
    """The prefix is taken away again before the chain: attention, positions, weights and evictions go by the own caches
    alone, every stage against the oracle."""
    from paper_2412_00061_b200.step import to_device
    from tests.parity_util import tolerances
    cfg, n_steps, budget = SHAPES[name], 5, 16
    step, s = _chain(cfg, n_steps, budget, decay=0.9)
    step.set_inputs(Kp=None, Vp=None)
    c, cache, n = step.chain, step.cache, cfg.max_nodes
    tol, scale = tolerances(cfg.dtype)[0], 1.0 / math.sqrt(cfg.D)
    none, nothing = np.zeros((cfg.Hkv, 0, cfg.D)), np.zeros(cfg.B, dtype=np.int64)
    K, V = np.array(s["K0"], copy=True), np.array(s["V0"], copy=True)
    kv, ev = s["kv_len0"].astype(np.int64), nothing.copy()
    mass, pos = np.zeros((cfg.B, cfg.Hkv, K.shape[2])), np.tile(np.arange(K.shape[2]), (cfg.B, cfg.Hkv, 1))
    c["kv_len"].copy_(c["kv_len0"])
    for t in range(n_steps):
        step.chain_head(t)
        n_nodes, mask = step.host("n_nodes").astype(np.int64), step.host("mask").view(np.uint64)
        np.testing.assert_array_equal(step.host("pos")[:, 0], ev + kv)
        hn, _ = synth.gen_node_hidden(cfg, synth.chain_step_seed(4, t), s["Wl"], step.host("node_tok"), step.host("parent"), n_nodes)
        c["hntab"][t].copy_(to_device(hn, cfg.dtype, step.device))
        step.chain_tail(t)
        step.check_status()
        for b in range(cfg.B):
            K[b, :, kv[b]:kv[b] + n], V[b, :, kv[b]:kv[b] + n] = s["Ktab"][t][b], s["Vtab"][t][b]
        O, lse = orc.tree_attention_shared(s["Qtab"][t], none, none, nothing, K, V, kv, n_nodes, mask, scale)
        assert np.max(np.abs(step.host("O") - O)) <= tol
        got_lse, fin = step.host("attn_lse"), np.isfinite(lse)
        assert np.array_equal(np.isfinite(got_lse), fin) and np.max(np.abs(got_lse[fin] - lse[fin])) <= 3e-4
        acc_len, acc_nodes = step.host("acc_len"), step.host("acc_nodes")
        K, V, kv, _ = orc.commit_accepted(K, V, kv, acc_len, acc_nodes, n)
        m, p = orc.attention_mass(s["Qtab"][t], K, kv, acc_len, acc_nodes, got_lse, scale, 0.9, mass, pos, ev)
        K, V, m, p, kv, ev = orc.evict_rows(K, V, m, p, kv, ev, budget, 3, 8)
        np.testing.assert_array_equal(c["kv_len"].cpu().numpy(), kv)
        np.testing.assert_array_equal(cache["n_evicted"].cpu().numpy(), ev)
        Kg, Vg = step.inp["K"].float().cpu().numpy(), step.inp["V"].float().cpu().numpy()
        got_m, got_p = cache["mass"].cpu().numpy(), cache["row_pos"].cpu().numpy()
        for b in range(cfg.B):
            L = int(kv[b])
            np.testing.assert_array_equal(got_p[b, :, :L], p[b, :, :L])
            np.testing.assert_allclose(got_m[b, :, :L], m[b, :, :L], rtol=2e-4, atol=1e-9)
            assert np.array_equal(Kg[b, :, :L], K[b, :, :L]) and np.array_equal(Vg[b, :, :L], V[b, :, :L])
        K, V, mass, pos = Kg.copy(), Vg.copy(), got_m.astype(np.float64), got_p.astype(np.int64)
    assert ev.max() > 0
