"""The draft head over 4-bit weights, against float64 products with the values that the weights stand for.

Tolerances.  A logit is a float32 sum of exact products (bfloat16 values; float32: products rounded by 2^-24).  bfloat16: a chain of
additions runs over the H / 256 16-element products of one of 8 warps and one of two accumulators, then 8 warps are added; each
addition is off by 2^-23 of the sum of magnitudes at most (tensor cores may truncate), so by (H/256 + 12) 2^-23 sum|x w| together.
float32: a lane's chain holds H/32 products (half a step, 2^-24, for product and addition together), then 2 + 8 additions:
(H/32 + 12) 2^-24 sum|x w|.  The log-sum-exp moves by the largest such error, and its own exponentials and sums (2^-21 each over a
few thousand additions of positive terms, chains of V/16/148 or more) stay below 2e-5; bound 3e-5 more."""
import numpy as np
import pytest
import torch

import q4_util as u

pytestmark = pytest.mark.gpu


class _Case:
    def __init__(self, dtype, M, H, V, T, k, group, mapped=False, bias=True, seed=0, B=None, weights=None):
        rng = np.random.default_rng([seed, M, H, V])
        act = u.act_of(dtype)
        self.dims = (dtype, M, H, V, T, k, group)
        self.h = u.handle(dtype, B=B or M, H=H, V=V, T=T, k=k, rows=M)
        rows = 3 * M if mapped else M
        self.x = torch.from_numpy(rng.normal(size=(rows, H)).astype(np.float32)).to(u.DEV, act)
        w = rng.normal(size=(T, V + 1, H)) * 0.05 if weights is None else weights
        self.W = torch.from_numpy(w.astype(np.float32)).to(u.DEV, act)
        self.x_rows = u.i32(rng.permutation(rows)[:M]) if mapped else None
        self.row_seq = u.i32(rng.integers(0, B, M)) if B else None
        self.bias = torch.from_numpy(rng.integers(0, 4, B or M).astype(np.float32)).to(u.DEV) if bias else None
        self.Wq = self.h.quantize_weights_q4(self.W, group)
        f32 = dict(dtype=torch.float32, device=u.DEV)
        self.out = [torch.full((M, T, k), -7, dtype=torch.int32, device=u.DEV), torch.zeros(M, T, k, **f32), torch.zeros(M, T, **f32)]
        self.z = torch.full((M, T, V + 1), 77.0, **f32)

    def run(self, dbg=True, **kw):
        self.h.draft_logits_q4(self.x, self.x_rows, self.Wq, self.row_seq, self.bias, *self.out, self.z if dbg else None, **kw)

    def reference(self):
        dtype, M, H, V, T, k, group = self.dims
        w = u.stands_for(self.W, group, dtype).to(u.DEV)
        x = (self.x if self.x_rows is None else self.x[self.x_rows.long()]).double()
        z = torch.einsum("mh,tvh->mtv", x, w)
        size = torch.einsum("mh,tvh->mtv", x.abs(), w.abs())
        if self.bias is not None:
            b = self.bias if self.row_seq is None else self.bias[self.row_seq.long()]
            z[:, :, V] += b.double()[:, None]
        err = (H / 256 + 12) * 2.0 ** -23 if dtype == "bf16" else (H / 32 + 12) * 2.0 ** -24
        return z, err * size + 2.0 ** -23 * z.abs()

    def check(self):
        dtype, M, H, V, T, k, group = self.dims
        assert self.h.poll_status() == 0
        z, tol = self.reference()
        assert torch.all((self.z.double() - z).abs() <= tol)
        # the selection, from the kernel's own logits: best first, ties to the lower id
        vals, ids = self.z.sort(dim=-1, descending=True, stable=True)
        assert torch.equal(self.out[0].long(), ids[..., :k])
        lse = torch.logsumexp(z, -1)
        assert torch.all((self.out[2].double() - lse).abs() <= tol.amax(-1) + 3e-5)
        assert torch.all((self.out[1] - (vals[..., :k] - self.out[2][..., None])).abs() <= 2e-6 * (1 + vals[..., :k].abs()))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,H,V,T,k,group", [
    (1, 8, 3, 1, 1, 32),            # the smallest
    (1, 256, 1000, 4, 3, 64),
    (3, 136, 97, 2, 5, 128),        # a short last group, a panel of one class
    (5, 1000, 333, 3, 2, 32),
    (8, 2048, 500, 2, 8, 64),
    (9, 520, 47, 8, 8, 128),        # two passes in float32 and more, a second tile in bfloat16
    (17, 4096, 130, 2, 4, 128),
])
def test_logits_selection_and_lse(dtype, M, H, V, T, k, group):
    c = _Case(dtype, M, H, V, T, k, group)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,M,H,V,group", [("bf16", 2, 10240, 200, 32), ("bf16", 12, 5120, 300, 64), ("bf16", 20, 8192, 64, 128), ("fp32", 5, 8192, 60, 64),
                                               ("fp32", 2, 10240, 40, 32), ("bf16", 33, 1536, 2500, 128), ("bf16", 70, 1088, 777, 64),
                                               ("bf16", 130, 72, 400, 32), ("bf16", 9, 64, 3, 32), ("bf16", 64, 4096, 3000, 128)])
def test_long_rows_and_several_passes(dtype, M, H, V, group):
    c = _Case(dtype, M, H, V, 2, 4, group, mapped=True)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_wide_vocabulary_with_rows_of_a_few_sequences(dtype):
    c = _Case(dtype, 6, 128, 50000, 3, 4, 32, B=2)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_equal_classes_rank_by_id(dtype):
    rng = np.random.default_rng(5)
    w = np.repeat(rng.normal(size=(2, 20, 64)), 20, axis=1)[:, :391]
    c = _Case(dtype, 3, 64, 390, 2, 7, 32, bias=False, weights=w)
    c.run()
    c.check()


def test_packed_weights_are_laid_out_as_described():
    H, V, T, group = 200, 20, 2, 64
    c = _Case("bf16", 1, H, V, T, 1, group)
    q, s, o = u.orc.q4_quantize(c.W.float().cpu().numpy(), group)
    words = c.Wq["w"].cpu().numpy().view("<u4").reshape(T, 2, 2, (1024 + 128) // 4)
    for t in range(T):
        for v in range(32):
            for h0 in range(0, 256, 8):
                panel, r, kb, e = v // 16, v % 16, h0 // 128, h0 % 128
                w = int(words[t, panel, kb, 64 * (e // 32) + 4 * r + e % 32 // 8])
                got = [((w | w << 32) >> bit) & 15 for bit in u.WORD_BITS]
                want = list(q[t, v, h0:h0 + 8]) if v <= V and h0 < H else [0] * 8
                assert got == want
                so = int(words[t, panel, kb, 256 + r * 2 + e // 64])
                there = v <= V and (h0 // 64) < s.shape[-1]
                pair = [np.array([x], dtype="<u4").view("<f4")[0] for x in ((so & 0xffff) << 16, so & 0xffff0000)]
                assert pair == ([s[t, v, h0 // 64], o[t, v, h0 // 64]] if there else [0.0, 0.0])


def test_a_row_map_that_leaves_x_is_reported_and_drafts_from_zeros():
    c = _Case("bf16", 3, 128, 40, 2, 2, 32, mapped=True, bias=False)
    c.x_rows[1] = 9
    c.run()
    assert c.h.poll_status() == -1
    assert torch.count_nonzero(c.z[1]) == 0 and torch.count_nonzero(c.z[2]) > 0


def test_replayed_and_on_another_stream():
    c = _Case("bf16", 4, 1024, 3001, 2, 3, 64)
    c.run()
    c.check()
    want = [t.clone() for t in c.out]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.run(dbg=False)
    for _ in range(3):
        for t in c.out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(c.out, want))
    for t in c.out:
        t.zero_()
    s.wait_stream(torch.cuda.current_stream())
    c.run(dbg=False, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(c.out, want))


def test_packing_may_directly_precede_the_draft():
    c = _Case("bf16", 1, 4096, 3000, 3, 4, 128)
    for seed in range(3):
        c.W.normal_(0.0, 0.05)
        c.Wq = c.h.quantize_weights_q4(c.W, 128)
        c.run()
        c.check()


def test_refusals():
    c = _Case("bf16", 2, 128, 40, 2, 2, 32)
    bad = u.binding.CtcsdError
    with pytest.raises(bad):
        c.h.quantize_weights_q4(c.W, 48)
    with pytest.raises(bad):
        c.h.quantize_weights_q4(c.W.float(), 32)
    with pytest.raises(bad):
        c.h.draft_logits_q4(c.x, None, dict(w=c.Wq["w"], group=64), None, c.bias, *c.out)      # packed with another group
    with pytest.raises(bad):
        c.h.draft_logits_q4(torch.cat([c.x, c.x]), None, c.Wq, None, c.bias, *c.out)           # more rows than the handle has room for
    with pytest.raises(bad):
        c.h.draft_logits_q4(c.x.t(), None, c.Wq, None, c.bias, *c.out)
    big = u.handle("fp32", B=1, H=65536, V=30, T=1, k=1)
    W = torch.zeros(1, 31, 65536, device=u.DEV)
    with pytest.raises(bad, match="unsupported"):
        big.draft_logits_q4(W[0, :1].contiguous(), None, big.quantize_weights_q4(W, 128), None, None, torch.zeros(1, 1, 1, dtype=torch.int32, device=u.DEV),
                            torch.zeros(1, 1, 1, device=u.DEV), torch.zeros(1, 1, device=u.DEV))
