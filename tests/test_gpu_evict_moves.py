"""Eviction where a CTA has a (sequence, kv head) to itself and moves about as many rows as its lists in shared memory hold
(2048): at the limit, one more, and few.  The kept rows are computed here by a sort; everything is exact."""
import numpy as np
import pytest

from test_gpu_cache_ops import _dev, _handle


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_lists_of_moves_at_the_limit_of_shared_memory(in_place):
    import torch
    B, Hkv, D, Lcap, budget, sinks, recent = 3, 80, 64, 5100, 3000, 4, 10
    kv = np.array([budget + 2048, budget + 2049, budget + 5], dtype=np.int32)
    rng = np.random.default_rng(41)
    mass = rng.random((B, Hkv, Lcap)).astype(np.float32)
    mass[:, :, budget:] += 10.0                                       # every row behind the new length stays
    pos = np.tile(np.arange(Lcap, dtype=np.int32), (B, Hkv, 1))
    ev = np.array([7, 0, 1], dtype=np.int32)
    K = torch.randn(B, Hkv, Lcap, D, device="cuda:0").to(torch.bfloat16)
    V = torch.randn(B, Hkv, Lcap, D, device="cuda:0").to(torch.bfloat16)
    K0, V0 = K.clone(), V.clone()
    h = _handle(B, Hkv, Hkv, D, "bf16")
    md, pd, kd, ed = _dev(mass), _dev(pos), _dev(kv), _dev(ev)
    outs = (md, pd, kd, ed) if in_place else (torch.full_like(md, -3.0), torch.full_like(pd, -3), torch.zeros_like(kd), torch.zeros_like(ed))
    h.evict_rows(h.make_eviction(Lcap), K, V, md, pd, kd, ed, budget, sinks, recent, *outs)
    assert h.poll_status() == 0
    assert outs[2].tolist() == [budget] * B and outs[3].tolist() == [7 + 2048, 2049, 1 + 5]
    got_pos, got_mass = outs[1].cpu().numpy(), outs[0].cpu().numpy()
    for b in range(B):
        L = int(kv[b])
        j = np.arange(L)
        safe = (j < sinks) | (j >= int(ev[b]) + L - recent)
        for g in range(0, Hkv, 7):
            kept = np.zeros(L, dtype=bool)
            kept[np.lexsort((j, -mass[b, g, :L], ~safe))[:budget]] = True
            src = np.arange(budget)
            src[~kept[:budget]] = budget + np.nonzero(kept[budget:])[0]
            np.testing.assert_array_equal(got_pos[b, g, :budget], src)
            np.testing.assert_array_equal(got_mass[b, g, :budget], mass[b, g, src])
            at = torch.from_numpy(src).to("cuda:0")
            assert torch.equal(K[b, g, :budget], K0[b, g][at]) and torch.equal(V[b, g, :budget], V0[b, g][at])
