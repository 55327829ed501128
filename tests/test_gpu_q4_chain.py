"""The 4-bit operators together, as a batch uses them: prompts stored in a 4-bit cache, then chained draft-and-verify steps (draft head over
4-bit weights -> tree -> attention over the 4-bit cache -> acceptance -> history update into it), every stage against the
oracle fed the GPU's output of the stage before.

Tolerances: attention as in test_gpu_q4_attention.py; cached rows, lengths and rows exact; log-probabilities as in test_gpu_q4_draft.py (H = 256:
below 1e-4 for these weights)."""
import math

import numpy as np
import pytest
import torch

import q4_util as u
from paper_2412_00061_b200 import synth

pytestmark = pytest.mark.gpu

C = synth.CONFIGS
SHAPES = {
    "mha": C["c2"].replace(name="mha", B=2, H=256, V=999, Hq=4, Hkv=4, kv_lo=30, kv_hi=300, max_nodes=32),
    "gqa_beam": C["c5"].replace(name="gqa_beam", B=11, H=256, V=800, Hq=8, Hkv=2, kv_lo=20, kv_hi=150, beam=16),
    "fp32": C["c1"].replace(name="fp32", B=2, H=128, V=300, kv_lo=5, kv_hi=40),
}


def _chain(cfg, n_steps, layout, group, seed=4):
    from paper_2412_00061_b200.step import DraftVerifyStep, to_device
    big = synth.chain_cache_config(cfg, n_steps)
    x0, Wd, bb = synth.gen_draft(cfg, seed)
    base_tok0, kv_len0 = synth.gen_base(cfg, seed)
    _, K0, V0 = synth.gen_attention(big, seed)
    Wl = synth.gen_lm_head(cfg, seed)
    Qtab, Ktab, Vtab = synth.gen_chain_tables(cfg, seed, n_steps)
    step = DraftVerifyStep(cfg, layout=layout)
    dev = step.device
    act = u.act_of(cfg.dtype)
    td = lambda a: to_device(a, cfg.dtype, dev)
    step.set_inputs(Wd=td(Wd), blank_bias=torch.from_numpy(bb).to(dev), Wl=td(Wl))
    step.quantize_draft_weights(group)
    step.set_inputs(Wd=None)
    cache = step.use_q4_cache(big.Lcap)
    step.store_prompt(td(K0), td(V0), u.i32(kv_len0))
    hntab = torch.zeros(n_steps, cfg.B * cfg.max_nodes, cfg.H, dtype=act, device=dev)
    step.setup_chain(n_steps, td(x0), u.i32(base_tok0), u.i32(kv_len0), td(Qtab), td(Ktab), td(Vtab), hntab)
    return step, cache, dict(Wd=Wd, bb=bb, Wl=Wl, K0=K0, V0=V0, x0=x0, kv_len0=kv_len0)


def _cache_values(step, cache, rows):
    cfg = step.cfg
    out = [torch.empty(cfg.B, cfg.Hkv, rows, cfg.D, dtype=u.act_of(cfg.dtype), device=step.device) for _ in range(2)]
    step.h.load_rows_q4(cache, None, u.i32([rows] * cfg.B), *out)
    return [t.double() for t in out]


@pytest.mark.parametrize("layout", ["packed", "raw"])
@pytest.mark.parametrize("name", sorted(SHAPES))
def test_chained_steps_in_4_bits(name, layout):
    from paper_2412_00061_b200.step import to_device
    cfg = SHAPES[name].replace(beam=0, T=4, k=3) if layout == "raw" else SHAPES[name]
    n_steps, group = 4, 64
    step, cache, s = _chain(cfg, n_steps, layout, group)
    c = step.chain
    Lcap = cache["Kq"].shape[2]
    K, V = (u.stands_for(torch.from_numpy(s[k]), 32, cfg.dtype).to(step.device) for k in ("K0", "V0"))
    W = u.stands_for(torch.from_numpy(s["Wd"]), group, cfg.dtype).to(step.device)
    kv = s["kv_len0"].astype(np.int64)
    c["kv_len"].copy_(c["kv_len0"])
    x = c["x0"].double()
    accepted = 0
    for t in range(n_steps):
        step.chain_head(t)
        step.check_status()
        z = torch.einsum("mh,tvh->mtv", x, W)
        z[:, :, -1] += torch.from_numpy(s["bb"]).to(step.device).double()[:, None]
        best = z.sort(dim=-1, descending=True).values[..., :cfg.k]
        ids = step.out["topk_id"].long()
        assert torch.all((z.gather(2, ids) - best).abs() <= 1e-4)
        assert torch.all((step.out["topk_lp"].double() - (best - torch.logsumexp(z, -1)[..., None])).abs() <= 2e-4)
        n_nodes, mask = step.host("n_nodes").astype(np.int64), step.host("mask").view(np.uint64)
        assert np.array_equal(step.host("pos")[:, 0], kv)
        parent = step.host("parent") if layout == "packed" else np.where(step.host("kept") != 0, step.host("nka"), -1)
        hn, _ = synth.gen_node_hidden(cfg, synth.chain_step_seed(4, t), s["Wl"], step.host("node_tok"), parent, n_nodes)
        c["hntab"][t].copy_(to_device(hn, cfg.dtype, step.device))
        step.chain_tail(t)
        step.check_status()
        Kt, Vt = c["Ktab"][t], c["Vtab"][t]
        O, lse = u.attention_reference(c["Qtab"][t], K, V, Kt, Vt, kv, n_nodes, mask, 1.0 / math.sqrt(cfg.D))
        vmax = 6.5
        tol = 2.0 ** -8 * (vmax + O.abs()) + 2e-4 * vmax if cfg.dtype == "bf16" else 2e-4 * vmax
        assert torch.all((step.out["O"].double() - O).abs() <= tol)
        there = torch.isfinite(lse)
        assert torch.all((step.out["attn_lse"].double() - lse)[there].abs() <= 2e-4 + 2.0 ** -22 * lse[there].abs())
        acc_len, acc_nodes = step.host("acc_len"), step.host("acc_nodes")
        accepted += int(acc_len.sum())
        sel = step.host("next_sel_row")
        for b in range(cfg.B):
            at = [0] + list(acc_nodes[b, :acc_len[b]])
            for dst, src in ((K, Kt), (V, Vt)):
                dst[b, :, kv[b]:kv[b] + len(at)] = u.stands_for(src[b][:, at], 32, cfg.dtype).to(step.device)
            assert sel[b] == b * cfg.max_nodes + at[-1]
        kv = kv + 1 + acc_len
        assert np.array_equal(c["kv_len"].cpu().numpy(), kv)
        got = _cache_values(step, cache, Lcap)
        for b in range(cfg.B):
            assert torch.equal(got[0][b, :, :kv[b]], K[b, :, :kv[b]]) and torch.equal(got[1][b, :, :kv[b]], V[b, :, :kv[b]])
        x = c["hntab"][t].double()[torch.from_numpy(sel.astype(np.int64)).to(step.device)]
    assert accepted > 0


@pytest.mark.parametrize("name", ["gqa_beam", "mha"])
def test_the_chain_again_and_in_a_graph(name):
    """Every run of the chain begins at its start; captured and replayed it gives the same."""
    step, cache, s = _chain(SHAPES[name], 3, "packed", 128)
    c = step.chain
    step.plant_chain_hidden(4, s["Wl"])
    step.run_chain()
    step.check_status()
    keep = lambda: [c["kv_len"].clone()] + [c["rec"][k].clone() for k in ("next_tok", "acc_len", "acc_nodes", "O", "topk_id")]
    want = keep()
    assert int(c["rec"]["acc_len"].sum()) > 0
    step.run_chain()
    assert all(torch.equal(a, b) for a, b in zip(keep(), want))
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step.run_chain()
    for _ in range(2):
        for t in c["rec"].values():
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        step.check_status()
        assert all(torch.equal(a, b) for a, b in zip(keep(), want))


def test_two_handles_side_by_side():
    """Steps of two handles on streams of their own, each with its workspace, give what they give one after the other."""
    made = [_chain(SHAPES[n], 2, "packed", 32, seed=6) for n in ("mha", "gqa_beam")]
    want = []
    for step, _, s in made:
        step.plant_chain_hidden(6, s["Wl"])
        step.run_chain()
        torch.cuda.synchronize()
        want.append([step.chain["rec"][k].clone() for k in ("O", "acc_len", "next_tok")])
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(3):
        for st, (step, _, _) in zip(streams, made):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                step.run_chain()
        torch.cuda.synchronize()
        for (step, _, _), w in zip(made, want):
            assert all(torch.equal(step.chain["rec"][k], t) for k, t in zip(("O", "acc_len", "next_tok"), w))
