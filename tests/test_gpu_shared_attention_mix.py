"""Shared-prefix tree attention where one warp's query rows belong to several sequences: whole blocks of keys that some rows
see and others do not, bad caches among good ones, and drawn shapes.  Inputs, checks and tolerances as in
test_gpu_shared_attention.py."""
import math

import numpy as np
import pytest

from test_gpu_shared_attention import _Run, _check, _inputs, _oracle, _poison_hidden


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, 3e38])
@pytest.mark.parametrize("nodes", [1, 20])
def test_a_bad_cache_of_many_blocks_stays_its_own(nodes, bad, dtype):
    """Sequences 1 and 4 hold NaN, infinities or the largest finite values in every row of a cache of several blocks;
    their neighbours, whose rows share a warp with theirs, are as the oracle has them."""
    rng = np.random.default_rng([31, nodes])
    B, Hq, Hkv, D = 6, 4, 2, 128
    x = _inputs(rng, B, Hq, Hkv, D, dtype, max(nodes, 2), [nodes] * B, [200, 300, 256, 0, 300, 128], [300, 513, 128, 640, 384, 5])
    want = _oracle({k: v.copy() for k, v in x.items()}, 1.0 / math.sqrt(D))
    for b in (1, 4):
        x["V"][b] = bad
        if not np.isfinite(bad):
            x["K"][b] = bad
    O, lse = _Run(x, dtype)().host()
    for b in (0, 2, 3, 5):
        _check(O[b], lse[b], want[0][b], want[1][b], dtype)
    if np.isfinite(bad):                         # finite values stay finite: the weights add up to 1
        assert np.all(np.isfinite(lse[[1, 4], :nodes]))
    else:
        assert not np.any(np.isfinite(O[[1, 4], :nodes]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("seed", range(10))
def test_drawn_shapes(seed, dtype):
    rng = np.random.default_rng([32, seed])
    D = int(rng.choice([64, 128]))
    Hkv = int(rng.choice([1, 2, 4]))
    grp = int(rng.choice([1, 2, 5, 8]))
    B = int(rng.integers(1, 13))
    nodes = int(rng.choice([2, 7, 33, 64]))
    live = rng.integers(0, nodes + 1, B)
    top = int(rng.choice([0, 90, 700]))
    pre = rng.integers(0, top + 1, B) if rng.integers(0, 2) else np.full(B, top)
    kv = rng.integers(0, int(rng.choice([3, 200, 900])) + 1, B)
    x = _inputs(rng, B, Hkv * grp, Hkv, D, dtype, nodes, live, pre, kv, Pcap=top)
    _poison_hidden(x)
    run = _Run(x, dtype)
    O, lse = run().host()
    _check(O, lse, *_oracle(x, run.scale), dtype)
