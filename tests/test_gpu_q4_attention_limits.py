"""Attention over a 4-bit cache at limits of its copies: the array's very last row where it stands alone behind a 16-byte boundary (heads
of 64, an odd number of rows), and batches whose plan leaves room for a few blocks in flight only.  Cases, reference and tolerances are those of
test_gpu_q4_attention.py."""
import numpy as np
import pytest
import torch

import q4_util as u
import test_gpu_q4_attention as attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,nodes", [(2, 3), (3, 40), (3, 100)])      # 16 query rows of a kv head at most, tiles of 128 and of 256
@pytest.mark.parametrize("B,Hkv,Lcap", [(1, 1, 1), (1, 1, 193), (3, 1, 129), (1, 3, 577), (1, 1, 3), (5, 1, 65)])
def test_an_odd_cache_that_is_full(Hq, nodes, B, Hkv, Lcap):
    c = attention._Case("bf16", B, Hq * Hkv, Hkv, 64, nodes, [nodes] * B, [Lcap] * B, Lcap=Lcap)
    for _ in range(3):
        c.run()
        c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B", [1024, 700])
def test_a_large_batch_of_trees_of_large_heads(dtype, B):
    rng = np.random.default_rng(B)
    nodes = 33
    n, kv = np.minimum(nodes, rng.integers(0, 7, B) ** 2), rng.integers(0, 300, B)
    n[5], n[-1], kv[-1] = nodes, nodes, 301
    c = attention._Case(dtype, B, 8, 1, 128, nodes, n, kv)
    c.run()
    c.check()
