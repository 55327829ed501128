"""A chain with a cache budget, run several times over (the walk that plants the hidden states, run_chain() twice, a graph
replayed twice, and once more on refilled rows): every run begins at the chain's start and gives the same tokens, positions,
outputs, caches and weights.  The first walk's stages are compared with the oracle in test_gpu_cache_chain.py; here its positions are counted
from the recorded lengths and its first attention is compared with the oracle on the start's rows (tolerances as there)."""
import math

import numpy as np
import pytest

from oracle import ctcsd_oracle as orc
from test_gpu_cache_chain import SHAPES, _chain

pytestmark = pytest.mark.gpu

RECORDED = ("node_tok", "pos", "O", "acc_len", "acc_tok", "next_tok", "new_kv_len")


def _left(step):
    k = step.cache
    return [t.clone() for t in (step.inp["K"], step.inp["V"], k["mass"], k["row_pos"], k["n_evicted"], step.chain["kv_len"])] + \
           [step.chain["rec"][n].clone() for n in RECORDED]


def _same(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("layout", ["packed", "raw"])
@pytest.mark.parametrize("name", sorted(SHAPES))
def test_every_run_begins_at_the_start(name, layout):
    import torch
    from tests.parity_util import tolerances
    cfg = SHAPES[name].replace(beam=0, T=4, k=3) if layout == "raw" else SHAPES[name]
    n_steps, budget = 5, 16
    step, s = _chain(cfg, n_steps, budget, layout)
    step.plant_chain_hidden(4, s["Wl"])
    first = _left(step)
    c, rec = step.chain, {k: step.chain["rec"][k].cpu().numpy().astype(np.int64) for k in ("pos", "acc_len", "new_kv_len", "n_nodes", "mask")}
    kv, ev = s["kv_len0"].astype(np.int64), np.zeros(cfg.B, dtype=np.int64)
    for t in range(n_steps):
        np.testing.assert_array_equal(rec["pos"][t][:, 0], s["pre"] + ev + kv)
        grown = kv + 1 + rec["acc_len"][t]
        kv = np.minimum(grown, budget)
        ev += grown - kv
        np.testing.assert_array_equal(rec["new_kv_len"][t], kv)
    assert ev.max() > 0
    for _ in range(2):
        step.run_chain()
        step.check_status()
        assert _same(_left(step), first)
    # the last run's first attention, on the start's rows
    K, V, kv0 = np.array(s["K0"], copy=True), np.array(s["V0"], copy=True), s["kv_len0"]
    for b in range(cfg.B):
        K[b, :, kv0[b]:kv0[b] + cfg.max_nodes] = s["Ktab"][0][b]
        V[b, :, kv0[b]:kv0[b] + cfg.max_nodes] = s["Vtab"][0][b]
    O, _ = orc.tree_attention_shared(s["Qtab"][0], s["Kp"], s["Vp"], s["pre"], K, V, kv0, rec["n_nodes"][0],
                                     c["rec"]["mask"][0].cpu().numpy().view(np.uint64), 1.0 / math.sqrt(cfg.D))
    assert np.max(np.abs(c["rec"]["O"][0].float().cpu().numpy() - O)) <= tolerances(cfg.dtype)[0]

    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step.run_chain()
        for _ in range(2):
            g.replay()
            side.synchronize()
            assert _same(_left(step), first)
        # other rows in the same buffers: from then on the graph begins with those
        other = -step.inp["K"].clone()
        step.inp["K"].copy_(other)
        step.reset_cache()
        step.save_chain_start()
        after = []
        for _ in range(2):
            g.replay()
            side.synchronize()
            after.append(_left(step))
        assert _same(after[0], after[1]) and not torch.equal(after[0][0], first[0])
    step.check_status()


def test_capturing_a_chain_that_has_no_start_is_refused():
    import torch
    from paper_2412_00061_b200 import binding
    step, s = _chain(SHAPES["gqa_beam"], 2, 50)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with pytest.raises(binding.CtcsdError):
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
                step.run_chain()
        step.save_chain_start()
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
            step.run_chain()
    torch.cuda.synchronize()
    step.check_status()
