"""The cache operators together, as a long-running batch uses them: chained draft-and-verify steps whose sequences share
a prefix and keep their caches within a budget (attention over prefix + own cache -> acceptance -> history update ->
gathered weight -> eviction), every stage against the oracle fed the GPU's output of the stage before.

Tolerances: attention outputs 2e-2 (bf16) / 2e-4 (fp32) max-abs and gathered weights 2e-4 relative, as derived in
test_gpu_shared_attention.py and test_gpu_cache_ops.py; integers, copied rows and positions exact."""
import math

import numpy as np
import pytest

from oracle import ctcsd_oracle as orc
from paper_2412_00061_b200 import synth
from tests.parity_util import tolerances

pytestmark = pytest.mark.gpu

C = synth.CONFIGS
SHAPES = {
    "mha": C["c2"].replace(name="mha", B=2, H=256, V=999, Hq=4, Hkv=4, kv_lo=30, kv_hi=60, max_nodes=32),
    "gqa_beam": C["c5"].replace(name="gqa_beam", B=3, H=256, V=800, Hq=8, Hkv=2, kv_lo=20, kv_hi=90, beam=16),
    "fp32": C["c1"].replace(name="fp32", B=2, H=128, V=300, kv_lo=5, kv_hi=40),
}


def _chain(cfg, n_steps, budget, layout="packed", prefix=37, seed=4, decay=0.9):
    import torch
    from paper_2412_00061_b200.step import DraftVerifyStep, to_device
    big = synth.chain_cache_config(cfg, n_steps)
    x0, Wd, bb = synth.gen_draft(cfg, seed)
    base_tok0, kv_len0 = synth.gen_base(cfg, seed)
    _, K0, V0 = synth.gen_attention(big, seed)
    Wl = synth.gen_lm_head(cfg, seed)
    Qtab, Ktab, Vtab = synth.gen_chain_tables(cfg, seed, n_steps)
    rng = np.random.default_rng(seed)
    Kp, Vp = (synth.to_dtype(rng.normal(size=(cfg.Hkv, prefix, cfg.D)).astype(np.float32), cfg.dtype) for _ in range(2))
    pre = np.array([prefix if b % 2 == 0 else prefix // 2 for b in range(cfg.B)], dtype=np.int32)
    step = DraftVerifyStep(cfg, layout=layout)
    dev = step.device
    i32 = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).to(dev)
    act = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
    step.set_inputs(Wd=to_device(Wd, cfg.dtype, dev), blank_bias=torch.from_numpy(bb).to(dev),
                    K=to_device(K0, cfg.dtype, dev), V=to_device(V0, cfg.dtype, dev), Wl=to_device(Wl, cfg.dtype, dev),
                    Kp=to_device(Kp, cfg.dtype, dev), Vp=to_device(Vp, cfg.dtype, dev), prefix_len=i32(pre))
    step.enable_cache_budget(budget, sinks=3, recent=8, decay=decay, Lcap=K0.shape[2])
    hntab = torch.zeros(n_steps, cfg.B * cfg.max_nodes, cfg.H, dtype=act, device=dev)
    step.setup_chain(n_steps, to_device(x0, cfg.dtype, dev), i32(base_tok0), i32(kv_len0), to_device(Qtab, cfg.dtype, dev),
                     to_device(Ktab, cfg.dtype, dev), to_device(Vtab, cfg.dtype, dev), hntab)
    return step, dict(Wl=Wl, K0=K0, V0=V0, Qtab=Qtab, Ktab=Ktab, Vtab=Vtab, Kp=Kp, Vp=Vp, pre=pre, kv_len0=kv_len0)


@pytest.mark.parametrize("layout", ["packed", "raw"])
@pytest.mark.parametrize("name", sorted(SHAPES))
def test_chained_steps_within_a_budget_behind_a_shared_prefix(name, layout):
    from paper_2412_00061_b200.step import to_device
    cfg = SHAPES[name].replace(beam=0, T=4, k=3) if layout == "raw" else SHAPES[name]
    n_steps, budget, decay = 6, 16, 0.9
    step, s = _chain(cfg, n_steps, budget, layout, decay=decay)
    c, cache = step.chain, step.cache
    tol, _ = tolerances(cfg.dtype)
    Kc, Vc = np.array(s["K0"], copy=True), np.array(s["V0"], copy=True)
    kv, ev = s["kv_len0"].astype(np.int64), np.zeros(cfg.B, dtype=np.int64)
    mass = np.zeros((cfg.B, cfg.Hkv, Kc.shape[2]))
    pos = np.tile(np.arange(Kc.shape[2]), (cfg.B, cfg.Hkv, 1))
    c["kv_len"].copy_(c["kv_len0"])
    n = cfg.max_nodes
    accepted = 0
    for t in range(n_steps):
        step.chain_head(t)
        step.check_status()
        n_nodes, mask = step.host("n_nodes").astype(np.int64), step.host("mask").view(np.uint64)
        # positions count the prefix, the dropped rows and the cached ones
        base = s["pre"] + ev + kv
        assert np.array_equal(step.host("pos")[:, 0], base)
        parent = step.host("parent") if layout == "packed" else np.where(step.host("kept") != 0, step.host("nka"), -1)
        hn, _ = synth.gen_node_hidden(cfg, synth.chain_step_seed(4, t), s["Wl"], step.host("node_tok"), parent, n_nodes)
        c["hntab"][t].copy_(to_device(hn, cfg.dtype, step.device))
        step.chain_tail(t)
        step.check_status()
        for b in range(cfg.B):
            Kc[b, :, kv[b]:kv[b] + n] = s["Ktab"][t][b]
            Vc[b, :, kv[b]:kv[b] + n] = s["Vtab"][t][b]
        O, lse = orc.tree_attention_shared(s["Qtab"][t], s["Kp"], s["Vp"], s["pre"], Kc, Vc, kv, n_nodes, mask, 1.0 / math.sqrt(cfg.D))
        # raw layout: a removed node's row sees kept ancestors only; every row is compared all the same
        assert np.max(np.abs(step.host("O") - O)) <= tol
        got_lse = step.host("attn_lse")
        fin = np.isfinite(lse)
        assert np.array_equal(np.isfinite(got_lse), fin) and np.max(np.abs(got_lse[fin] - lse[fin])) <= 3e-4
        acc_len, acc_nodes = step.host("acc_len"), step.host("acc_nodes")
        accepted += int(acc_len.sum())
        Kc, Vc, kv, _ = orc.commit_accepted(Kc, Vc, kv, acc_len, acc_nodes, n)
        want_m, want_p = orc.attention_mass(s["Qtab"][t], Kc, kv, acc_len, acc_nodes, got_lse, 1.0 / math.sqrt(cfg.D), decay, mass, pos, ev)
        # (the weights before the eviction are not visible from outside: the eviction is checked on the oracle's)
        Ke, Ve, me, pe, kve, eve = orc.evict_rows(Kc, Vc, want_m, want_p, kv, ev, budget, 3, 8)
        got_m, got_p = cache["mass"].cpu().numpy(), cache["row_pos"].cpu().numpy()
        np.testing.assert_array_equal(c["kv_len"].cpu().numpy(), kve)
        np.testing.assert_array_equal(cache["n_evicted"].cpu().numpy(), eve)
        Kg, Vg = step.inp["K"].float().cpu().numpy(), step.inp["V"].float().cpu().numpy()
        for b in range(cfg.B):
            L = int(kve[b])
            np.testing.assert_array_equal(got_p[b, :, :L], pe[b, :, :L])
            np.testing.assert_allclose(got_m[b, :, :L], me[b, :, :L], rtol=2e-4, atol=1e-9)
            assert np.array_equal(Kg[b, :, :L], Ke[b, :, :L]) and np.array_equal(Vg[b, :, :L], Ve[b, :, :L])
        Kc, Vc, mass, pos, kv, ev = Ke, Ve, got_m.astype(np.float64), got_p.astype(np.int64), kve, eve
        Kc, Vc = np.array(Kg, copy=True), np.array(Vg, copy=True)
    assert ev.max() > 0 and accepted > 0


def test_the_chain_in_a_graph_equals_the_chain():
    """run_chain() captured and replayed twice: the same tokens, caches, weights and positions as run eagerly."""
    import torch
    cfg = SHAPES["gqa_beam"]
    step, s = _chain(cfg, 4, 50)
    from paper_2412_00061_b200.step import to_device
    c, cache = step.chain, step.cache
    state = lambda: [step.inp["K"], step.inp["V"], cache["mass"], cache["row_pos"], cache["n_evicted"], c["kv_len"]]

    def reset():
        step.inp["K"].copy_(to_device(s["K0"], cfg.dtype, step.device))
        step.inp["V"].copy_(to_device(s["V0"], cfg.dtype, step.device))
        cache["mass"].zero_()
        cache["row_pos"].copy_(torch.arange(cache["row_pos"].shape[2], dtype=torch.int32, device=step.device).expand_as(cache["row_pos"]))
        cache["n_evicted"].zero_()

    step.plant_chain_hidden(4, s["Wl"])
    reset()
    step.run_chain()
    step.check_status()
    want = [t.clone() for t in state()] + [c["rec"][k].clone() for k in ("next_tok", "acc_len", "O")]
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        reset()
        with torch.cuda.graph(g, stream=side):
            step.run_chain()
        for _ in range(2):
            reset()
            g.replay()
            side.synchronize()
            got = state() + [c["rec"][k] for k in ("next_tok", "acc_len", "O")]
            for a, b in zip(got, want):
                assert torch.equal(a, b)
    step.check_status()


def test_two_streams_with_a_workspace_each():
    """Two handles with their own workspaces, their calls overlapping on two streams, give what they give alone."""
    import torch
    from tests.test_gpu_shared_attention import _Run, _inputs
    runs = [_Run(_inputs(np.random.default_rng(60 + k), 4, 8, 2, 128, "bf16", 32, [32, 9, 20, 1], [700] * 4, [300, 80, 0, 555]), "bf16") for k in range(2)]
    want = [[a.copy() for a in r().host()] for r in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for r, s in zip(runs, streams):
            with torch.cuda.stream(s):
                r()
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        O, lse = r.host()
        assert np.array_equal(O, w[0]) and np.array_equal(lse, w[1])


def test_offsets_past_32_bits():
    """Caches of more than 2^32 elements: the last sequence's last head lies behind every 32-bit offset."""
    import torch
    from paper_2412_00061_b200 import binding
    B, Hq, Hkv, D, nodes, T = 2, 4, 2, 128, 8, 3
    Lcap = (1 << 32) // (B * Hkv * D) + 4096
    rng = np.random.default_rng(70)
    h = binding.Handle(B, 64, 50, T, 2, 8, 4, nodes, Hq, Hkv, D, binding.DTYPE_BF16)
    dev, bf = "cuda:0", torch.bfloat16
    K = torch.zeros(B, Hkv, Lcap, D, dtype=bf, device=dev)
    V = torch.zeros_like(K)
    assert K.numel() > 1 << 32
    kv, n, far = 600, 5, Lcap - 700
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
    h.tree_attention_shared(h.make_shared_attention(), d(Q).to(bf), None, None, None, K, V, i32(kv, kv), i32(n, n), d(mask.view(np.int64)),
                            scale, O, lse)
    want_O, want_lse = orc.tree_attention_shared(Q, np.zeros((Hkv, 0, D)), np.zeros((Hkv, 0, D)), [0, 0], Ks, Vs, [kv, kv], [n, n], mask, scale)
    assert np.max(np.abs(O.float().cpu().numpy() - want_O)) <= 2e-2
    f = np.isfinite(want_lse)
    assert np.max(np.abs(lse.cpu().numpy()[f] - want_lse[f])) <= 3e-4
    # two accepted nodes behind the root; then rows far behind in the cache take part in an eviction
    mass = torch.zeros(B, Hkv, Lcap, device=dev)
    pos = torch.arange(Lcap, dtype=torch.int32, device=dev).repeat(B, Hkv, 1)
    path = np.tile(np.array([1, 2, -1], dtype=np.int32), (B, 1))
    h.attention_mass(d(Q).to(bf), K, i32(kv + 3, kv + 3), i32(2, 2), d(path), lse, scale, mass, pos)
    want_m, _ = orc.attention_mass(Q, Ks, np.array([kv + 3] * 2), np.array([2, 2]), path, lse.cpu().numpy(), scale, 1.0,
                                   np.zeros((B, Hkv, kv + n)), np.zeros((B, Hkv, kv + n), dtype=np.int64))
    np.testing.assert_allclose(mass[:, :, :kv + 3].cpu().numpy(), want_m[:, :, :kv + 3], rtol=2e-4, atol=1e-9)
    L, budget = far + 300, far + 290
    K[:, :, far:L], V[:, :, far:L] = d(r(B, Hkv, 300, D)).to(bf), d(r(B, Hkv, 300, D)).to(bf)
    mass.fill_(1.0)
    low = torch.tensor([5, far + 7, far + 100, L - 1], device=dev)
    mass[:, :, low] = 0.5
    mass[:, :, L - 6:L - 1] = 0.25                       # the ten that go: these five, then 0.5s and the last of the ones
    tail = K[:, :, L - 10:L].clone()
    kvd, ev = i32(L, L), i32(0, 0)
    h.evict_rows(h.make_eviction(Lcap), K, V, mass, pos, kvd, ev, budget, 0, 0, mass, pos, kvd, ev)
    assert h.poll_status() == 0
    assert kvd.tolist() == [budget] * 2 and ev.tolist() == [10] * 2
    # dropped: L-6..L-2 (0.25), 5, far+7, far+100, L-1 (0.5) and one of the ones: the highest row, L-7; kept behind the
    # budget: L-10, L-9, L-8, which fill 5, far+7, far+100
    for dst, src in zip([5, far + 7, far + 100], range(3)):
        assert torch.equal(K[:, :, dst], tail[:, :, src])
        assert pos[:, :, dst].unique().tolist() == [L - 10 + src]


def test_eviction_under_the_debug_bounds_build():
    """The build that checks the index of every store: no check may fail."""
    from paper_2412_00061_b200 import binding, build
    from tests import test_gpu_cache_ops as ops
    lib = binding.use_library(build.build(debug_bounds=True))
    try:
        assert lib.ctcsd_debug_bounds_enabled() == 1
        for name in ("to_one_row", "ragged", "half", "cluster"):
            ops.test_eviction(name, True, "bf16", True)          # (asserts a clean status word)
    finally:
        assert binding.use_library(None).ctcsd_debug_bounds_enabled() == 0
