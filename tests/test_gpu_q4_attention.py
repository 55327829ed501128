"""Tree attention over a 4-bit cache against float64 attention over the values that the cache stands for.

Tolerances.  Values |v| <= 5 or so (vmax below: the largest there is).  bfloat16: a weight is rounded to bfloat16 once for the product with V
(half a step, 2^-8 relative, at most), so a convex combination moves by 2^-8 vmax at most, and the result is rounded once (2^-8 |o|).
Scores are float32 sums of exact products: D additions of 2^-23 of sum|q k| scale <= 128 * 2^-23 * 2 sqrt(D) max|k| / 1 -> below 2e-3 for
these inputs (|k| <= 12), which moves weights, and so outputs, by 2e-3 vmax and the log-sum-exp by 2e-3.  The additions' errors are random
in sign; bounds used: 2^-8 vmax + 2^-8 |o| + 2e-4 vmax, and 2e-4 + 2^-22 |lse| for the log-sum-exp.
float32: 2e-4 vmax and 2e-4."""
import numpy as np
import pytest
import torch

import q4_util as u

pytestmark = pytest.mark.gpu


class _Case:
    def __init__(self, dtype, B, Hq, Hkv, D, nodes, n, kv, seed=0, Lcap=None):
        rng = np.random.default_rng([seed, B, Hq, D, nodes])
        act = u.act_of(dtype)
        self.dtype, self.D, self.nodes = dtype, D, max(2, nodes)
        self.n, self.kv = np.asarray(n), np.asarray(kv)
        Lcap = Lcap or max(1, int(self.kv.max())) + 5
        self.h = u.handle(dtype, B=B, nodes=nodes, Hq=Hq, Hkv=Hkv, D=D)
        gen = torch.Generator(device=u.DEV).manual_seed(seed * 31 + B)
        r = lambda *s: torch.randn(*s, generator=gen, device=u.DEV).clamp_(-5, 5)
        self.Q = r(B, self.nodes, Hq, D).to(act)
        self.K, self.V = (r(B, Hkv, Lcap, D) + 0.5 * r(D)).to(act), r(B, Hkv, Lcap, D).to(act)
        self.Kt, self.Vt = (r(B, Hkv, self.nodes, D) + 0.5 * r(D)).to(act), r(B, Hkv, self.nodes, D).to(act)
        self.mask = u.tree_mask(rng, B, nodes, self.n)
        self.cache = self.h.make_q4_cache(Lcap)
        self.h.store_rows_q4(self.cache, self.K, self.V, u.i32([Lcap] * B))
        self.ws = self.h.make_q4_attention()
        self.O = torch.full((B, self.nodes, Hq, D), 9.0, dtype=act, device=u.DEV)
        self.lse = torch.full((B, self.nodes, Hq), 9.0, device=u.DEV)
        self.lens = u.i32(self.kv), u.i32(self.n)
        self.mask_dev = torch.from_numpy(self.mask.view(np.int64)).to(u.DEV)
        self.scale = 1.0 / np.sqrt(D)

    def run(self, lse=True, **kw):
        self.h.tree_attention_q4(self.ws, self.Q, self.cache, self.Kt, self.Vt, *self.lens, self.mask_dev, self.scale, self.O, self.lse if lse else None, **kw)

    def values(self):
        return [torch.from_numpy(u.orc.q4_values(*u.orc.q4_quantize(t.float().cpu().numpy(), 32), 32, self.dtype == "bf16")).to(u.DEV) for t in (self.K, self.V)]

    def check(self, lse=True):
        assert self.h.poll_status() == 0
        K, V = self.values()
        O, L = u.attention_reference(self.Q, K, V, self.Kt, self.Vt, self.kv, self.n, self.mask, self.scale)
        vmax = 6.5
        if self.dtype == "bf16":
            tol = 2.0 ** -8 * (vmax + O.abs()) + 2e-4 * vmax
        else:
            tol = 2e-4 * vmax
        assert torch.all((self.O.double() - O).abs() <= tol)
        if lse:
            there = torch.isfinite(L)
            assert torch.equal(there, torch.isfinite(self.lse)) and torch.all(self.lse[~there] == -np.inf)
            assert torch.all((self.lse.double() - L)[there].abs() <= 2e-4 + 2.0 ** -22 * L[there].abs())


SHAPES = [
    # dtype-independent: B, Hq, Hkv, D, nodes, live nodes, cached rows
    (1, 1, 1, 64, 2, [1], [0]),                            # a key sees itself alone
    (1, 4, 4, 64, 32, [32], [128]),
    (2, 8, 1, 64, 2, [1, 2], [1, 257]),                    # single tokens, eight heads a kv head
    (3, 6, 2, 128, 7, [7, 0, 3], [0, 50, 129]),            # a sequence without nodes, one without a cache
    (2, 12, 3, 64, 33, [33, 17], [64, 63]),                # odd trees, lengths at a block's edge
    (2, 4, 1, 128, 64, [64, 40], [500, 127]),              # 256 rows of a kv head
    (1, 28, 4, 64, 100, [71], [777]),
    (2, 3, 1, 128, 256, [256, 129], [5, 300]),             # the largest tree, more than one block of tree rows
    (5, 5, 5, 128, 2, [1, 1, 1, 1, 1], [3000, 1, 0, 128, 2049]),
    (1, 16, 1, 128, 2, [2], [4097]),                       # 32 rows of a kv head
    (1, 64, 1, 64, 9, [8], [300]),                         # 512 rows
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,Hq,Hkv,D,nodes,n,kv", SHAPES)
def test_outputs_and_lse(dtype, B, Hq, Hkv, D, nodes, n, kv):
    c = _Case(dtype, B, Hq, Hkv, D, nodes, n, kv)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [1, 3, 5, 7, 8])
def test_what_is_hidden_does_not_count(dtype, shape):
    """NaN behind the lengths, in unused tree rows and queries, and in a branch that other nodes do not see."""
    B, Hq, Hkv, D, nodes, n, kv = SHAPES[shape]
    c = _Case(dtype, B, Hq, Hkv, D, nodes, n, kv, seed=3)
    c.run()
    plain = c.O.clone(), c.lse.clone()
    for b in range(B):
        for name in ("Ks", "Vs"):
            c.cache[name][b, :, kv[b]:] = float("nan")
        for t in (c.Kt, c.Vt):
            t[b, :, n[b]:] = float("nan")
        c.Q[b, n[b]:] = float("inf")
    c.run()
    assert c.h.poll_status() == 0
    assert torch.equal(c.O, plain[0]) and torch.equal(c.lse, plain[1])
    # a leaf's key and value become NaN and infinite: only the rows that see it may change
    b = int(np.argmax(c.n))
    leaf = int(c.n[b]) - 1
    sees = [(int(c.mask[b, i, leaf // 64]) >> (leaf % 64)) & 1 for i in range(int(c.n[b]))]
    c.Kt[b, :, leaf] = float("nan")
    c.Vt[b, :, leaf] = float("inf")
    c.run()
    assert c.h.poll_status() == 0
    for i, s in enumerate(sees):
        if not s:
            assert torch.equal(c.O[b, i], plain[0][b, i]) and torch.equal(c.lse[b, i], plain[1][b, i])
    assert sum(sees) >= 1


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_nodes_that_see_nothing(dtype):
    """Without a cache, a node whose mask is empty sees no key: zero and -inf."""
    c = _Case(dtype, 2, 4, 2, 64, 5, [5, 5], [0, 3])
    c.mask[:, 3] = 0
    c.mask_dev = torch.from_numpy(c.mask.view(np.int64)).to(u.DEV)
    c.run()
    c.check()
    assert torch.count_nonzero(c.O[0, 3]) == 0 and torch.all(c.lse[0, 3] == -np.inf) and torch.isfinite(c.lse[1, 3]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_scores(dtype):
    """Scores of hundreds, rising along the cache: the reference of the exponents has to follow."""
    c = _Case(dtype, 1, 2, 1, 64, 3, [3], [700])
    ramp = torch.linspace(-3, 3, c.K.shape[2], device=u.DEV)[None, None, :, None]
    c.K = (c.K.float() * 0.05 + ramp).to(c.K.dtype)
    c.Q = (c.Q.float() * 0.05 + 6.0).to(c.Q.dtype)
    c.h.store_rows_q4(c.cache, c.K, c.V, u.i32([c.K.shape[2]]))
    c.run()
    K, V = c.values()
    O, L = u.attention_reference(c.Q, K, V, c.Kt, c.Vt, c.kv, c.n, c.mask, c.scale)
    assert float(L.max()) > 100
    # scores of some 150 are sums of 64 products, each addition off by 2^-23 of 150 at most: 1.2e-3 for a score
    assert torch.all((c.lse.double() - L).abs() <= 1.2e-3)
    assert torch.all((c.O.double() - O).abs() <= (2.0 ** -8 * (6.5 + O.abs()) if dtype == "bf16" else 0) + 1.2e-3 * 2 * 6.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_lengths_outside_the_arrays_are_reported(dtype):
    c = _Case(dtype, 4, 2, 2, 64, 4, [2, 3, 4, 4], [5, 9, 7, 8], Lcap=9)
    c.lens = u.i32([5, 10, -1, 8]), u.i32([2, 3, 4, 5])
    c.run()
    assert c.h.poll_status() == -1
    assert torch.count_nonzero(c.O[1:]) == 0 and torch.all(c.lse[1:] == -np.inf)
    c.kv, c.n = np.array([5, 0, 0, 0]), np.array([2, 0, 0, 0])
    c.check()


def test_the_longest_sequence_may_fill_the_cache_and_no_lse_is_asked_for():
    c = _Case("bf16", 2, 4, 2, 128, 5, [5, 5], [300, 300], Lcap=300)
    c.run(lse=False)
    c.check(lse=False)
    assert torch.all(c.lse == 9.0)


def test_thousand_sequences():
    rng = np.random.default_rng(9)
    n, kv = rng.integers(0, 4, 1024), rng.integers(0, 40, 1024)
    c = _Case("bf16", 1024, 2, 1, 64, 3, n, kv)
    c.run()
    c.check()


def test_same_result_again_captured_and_on_another_stream():
    c = _Case("bf16", 3, 8, 2, 128, 64, [64, 20, 50], [1000, 37, 400])
    c.run()
    c.check()
    want = c.O.clone(), c.lse.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.run()
    for _ in range(3):
        c.O.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.O, want[0]) and torch.equal(c.lse, want[1])
    c.lens[0][1] = 300                                     # lengths are read on the device: the graph follows them
    c.kv[1] = 300
    g.replay()
    torch.cuda.synchronize()
    c.check()


def test_refusals():
    c = _Case("bf16", 1, 2, 1, 64, 3, [3], [7])
    bad = u.binding.CtcsdError
    args = lambda **k: [k.get("ws", c.ws), k.get("Q", c.Q), k.get("cache", c.cache), k.get("Kt", c.Kt), c.Vt, *c.lens, c.mask_dev, k.get("scale", c.scale), c.O]
    for k in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(Q=c.Q.float()), dict(Kt=c.Kt[:, :, :2]),
              dict(cache=dict(c.cache, Ks=c.cache["Ks"][:, :, :4].contiguous())), dict(ws=dict(c.ws, ws_bytes=c.ws["ws_bytes"] - 256)),
              dict(ws=dict(c.ws, ws_ptr=c.ws["ws_ptr"] + 16))):
        with pytest.raises(bad):
            c.h.tree_attention_q4(*args(**k))
