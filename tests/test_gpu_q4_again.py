"""Captured steps over 4-bit weights and a 4-bit cache, when another batch takes the cache's place and the weights are packed again: the graph
follows, as it gives what the same calls give uncaptured."""
import numpy as np
import pytest
import torch

import q4_util as u
from paper_2412_00061_b200 import synth
from paper_2412_00061_b200.step import to_device
from test_gpu_q4_chain import SHAPES, _chain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["mha", "gqa_beam", "fp32"])
def test_a_graph_follows_another_batch_in_the_same_cache(name):
    step, cache, s = _chain(SHAPES[name], 3, "packed", 64)
    c, cfg = step.chain, step.cfg
    step.plant_chain_hidden(4, s["Wl"])
    step.run_chain()
    first = c["rec"]["O"].clone()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        step.run_chain()
    # another prompt in the same cache, other weights in the same tensor
    big = synth.chain_cache_config(cfg, 3)
    _, K1, V1 = synth.gen_attention(big, 9)
    Wd = to_device(synth.gen_draft(cfg, 9)[1], cfg.dtype, step.device)
    step.inp["Wd"] = Wd                          # (the packed weights stay in use until they are packed again)
    packed, w = step.inp["Wd_q4"], step.inp["Wd_q4"]["w"]
    assert step.quantize_draft_weights(64) is packed and packed["w"] is w
    assert step.use_q4_cache(big.Lcap) is cache
    assert all(torch.count_nonzero(t) == 0 for t in cache.values())
    lens = np.maximum(1, s["kv_len0"] // 2)
    step.store_prompt(to_device(K1, cfg.dtype, step.device), to_device(V1, cfg.dtype, step.device), u.i32(lens))
    c["kv_len0"].copy_(u.i32(lens))
    junk = [torch.full_like(t, 1) for t in list(cache.values()) + [w] for _ in range(2)]       # (what was let go would be handed out here)
    step.run_chain()
    step.check_status()
    keep = ("next_tok", "acc_len", "acc_nodes", "O", "topk_id", "new_kv_len")
    want = [c["rec"][k].clone() for k in keep]
    assert not torch.equal(c["rec"]["O"], first)
    rows = [t.clone() for t in cache.values()]
    for _ in range(2):
        for t in c["rec"].values():
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        step.check_status()
        assert all(torch.equal(c["rec"][k], t) for k, t in zip(keep, want))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(cache.values(), rows))
    assert all(torch.all(t == 1) for t in junk)


def test_weights_packed_on_a_side_stream_and_let_go_at_once():
    """The side stream is behind, the weights are dropped, and their memory and more like it is written over on the current stream."""
    import test_gpu_q4_draft as draft
    c = draft._Case("bf16", 2, 1024, 4000, 2, 3, 64)
    c.run()
    want = [t.clone() for t in c.out]
    plain, packed = c.W, c.Wq["w"].clone()
    side = torch.cuda.Stream()
    for _ in range(3):
        W = plain.clone()
        busy = torch.full_like(packed, 3)                    # in use on the current stream when it is let go
        torch.cuda._sleep(20_000_000)
        busy.add_(1)
        del busy
        with torch.cuda.stream(side):
            torch.cuda._sleep(40_000_000)
        got = c.h.quantize_weights_q4(W, 64, stream=side)
        del W
        over = [torch.full_like(plain, float("nan")) for _ in range(2)]
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got["w"], packed)
        c.Wq = got
        c.run()
        assert all(torch.equal(a, b) for a, b in zip(c.out, want))
        del over, got
