"""Pins of the oracle's cache operators against facts that do not depend on how they are written."""
import math

import numpy as np
import torch

from oracle import ctcsd_oracle as orc


def _tree_mask(parent):
    n = len(parent)
    m = np.zeros((1, n, (n + 63) // 64), dtype=np.uint64)
    for i in range(n):
        j = i
        while j >= 0:
            m[0, i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
            j = parent[j]
    return m


def test_a_shared_prefix_equals_the_same_rows_in_every_cache():
    rng = np.random.default_rng(1)
    B, n, Hq, Hkv, D, P = 3, 5, 4, 2, 8, 7
    kv = np.array([0, 3, 6])
    nn = np.array([5, 1, 4])
    pre = np.array([7, 0, 4])
    Q = rng.normal(size=(B, n, Hq, D))
    Kp, Vp = rng.normal(size=(2, Hkv, P, D))
    K, V = rng.normal(size=(2, B, Hkv, 12, D))
    mask = np.repeat(_tree_mask([-1, 0, 0, 1, 2]), B, axis=0)
    O, lse = orc.tree_attention_shared(Q, Kp, Vp, pre, K, V, kv, nn, mask, 0.3)
    for b in range(B):
        p = pre[b]
        Kb = np.concatenate([Kp[:, :p], K[b]], axis=1)[None]
        Vb = np.concatenate([Vp[:, :p], V[b]], axis=1)[None]
        want = orc.tree_attention(Q[b:b + 1], Kb, Vb, kv[b:b + 1] + p, nn[b:b + 1], mask[b:b + 1], 0.3)
        np.testing.assert_allclose(O[b], want[0], rtol=1e-12, atol=1e-13)
    # the log-sum-exp normalises the weights: attention over values of one is one, over keys' own scores their mean
    x = torch.tensor(Q[0, 3, 1] @ np.concatenate([Kp[0], K[0, 0, :5]]).T * 0.3)
    vis = torch.tensor([True] * 7 + [True, True, False, True, False])
    assert abs(torch.logsumexp(x[vis], 0).item() - lse[0, 3, 1]) < 1e-12
    assert np.all(lse[1, 1:] == -np.inf) and np.all(O[1, 1:] == 0)


def test_gathered_weight_of_one_step_sums_to_the_number_of_queries():
    """Without a shared prefix a query's weights over its own rows sum to one, so the step adds (accepted + 1)
    x heads per kv head in total; rows before the root get the decayed old mass on top."""
    rng = np.random.default_rng(2)
    B, n, Hq, Hkv, D, T, Lcap = 2, 6, 6, 2, 8, 3, 40
    acc = np.array([0, 3])
    path = np.array([[-1, -1, -1], [1, 3, 5]])
    kv = np.array([1, 30])
    Q = rng.normal(size=(B, n, Hq, D))
    K = rng.normal(size=(B, Hkv, Lcap, D))
    lse = np.full((B, n, Hq), np.nan)
    for b in range(B):
        for l, node in enumerate([0] + list(path[b, :acc[b]])):
            for h in range(Hq):
                s = K[b, h // 3, :kv[b] - acc[b] + l] @ Q[b, node, h] * 0.5
                lse[b, node, h] = torch.logsumexp(torch.tensor(s), 0).item()
    m0 = rng.random((B, Hkv, Lcap))
    pos0 = np.full((B, Hkv, Lcap), -5)
    m, pos = orc.attention_mass(Q, K, kv, acc, path, lse, 0.5, 0.25, m0, pos0, np.array([10, 100]))
    for b in range(B):
        base = kv[b] - 1 - acc[b]
        added = m[b, :, :kv[b]].sum(-1) - 0.25 * m0[b, :, :base].sum(-1)
        np.testing.assert_allclose(added, (acc[b] + 1) * 3, rtol=1e-12)
        np.testing.assert_array_equal(pos[b, 0, base:kv[b]], [10, 100][b] + np.arange(base, kv[b]))
        assert np.array_equal(m[b, :, kv[b]:], m0[b, :, kv[b]:]) and np.all(pos[b, :, :base] == -5)
    # the last row is seen by the last query alone: its weight is that query's softmax there
    h = 4
    s = K[1, 1, :30] @ Q[1, 5, h] * 0.5
    one = sum(math.exp(K[1, 1, 29] @ Q[1, 5, hh] * 0.5 - lse[1, 5, hh]) for hh in (3, 4, 5))
    assert abs(one - m[1, 1, 29]) < 1e-12 and s.shape == (30,)


def test_eviction_by_hand():
    """Ten rows, budget 6, one sink, two newest: kept are position 0, the two newest and the three heaviest
    others, a tie going to the lower row; kept rows behind the budget fill the holes in order."""
    K = np.arange(10, dtype=np.float64).reshape(1, 1, 10, 1)
    pos = np.array([[[3, 0, 1, 4, 2, 5, 6, 7, 8, 9]]])
    mass = np.array([[[.5, .0, .9, .5, .1, np.nan, .5, .7, .0, .0]]])
    K1, V1, m1, p1, kv, ev = orc.evict_rows(K, -K, mass, pos, np.array([10]), np.array([0]), 6, 1, 2)
    # protected: row 1 (position 0), rows 8 and 9; then .9 (row 2), .7 (row 7), and of the three .5 the lowest row: 0
    assert K1[0, 0, :6, 0].tolist() == [0, 1, 2, 7, 8, 9]
    assert V1[0, 0, :6, 0].tolist() == [0, -1, -2, -7, -8, -9]
    assert p1[0, 0, :6].tolist() == [3, 0, 1, 7, 8, 9] and m1[0, 0, :6].tolist() == [.5, 0, .9, .7, 0, 0]
    assert kv.tolist() == [6] and ev.tolist() == [4]


def test_eviction_keeps_the_attention_of_what_is_kept():
    """Dropping rows and reordering the rest leaves attention over the kept rows as it is: the softmax over the
    new cache equals the softmax over the old one restricted to the kept rows."""
    rng = np.random.default_rng(3)
    L, D = 50, 4
    K, V = rng.normal(size=(2, 1, 1, L, D))
    mass = rng.random((1, 1, L))
    pos = rng.permutation(L).reshape(1, 1, L)
    K1, V1, m1, p1, kv, _ = orc.evict_rows(K, V, mass, pos, np.array([L]), np.array([0]), 20, 2, 5)
    kept = sorted(np.nonzero(np.isin(pos[0, 0], p1[0, 0, :20]))[0])
    assert len(kept) == 20
    q = rng.normal(size=D)
    a = np.exp(K[0, 0, kept] @ q)
    b = np.exp(K1[0, 0, :20] @ q)
    np.testing.assert_allclose((a / a.sum()) @ V[0, 0, kept], (b / b.sum()) @ V1[0, 0, :20], rtol=1e-12)
    worst_kept = min(m for m, p in zip(m1[0, 0, :20], p1[0, 0, :20]) if 2 <= p < 45)
    dropped = [mass[0, 0, j] for j in range(L) if j not in kept]
    assert worst_kept >= max(dropped)
