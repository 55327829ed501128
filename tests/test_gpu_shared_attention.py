"""GPU parity of shared-prefix tree attention against the oracle.

Tolerances.  bfloat16: an output is a convex combination of values |v| <= 5 here; every weight is rounded to
bfloat16 (2^-8 relative at most), so the combination moves by at most 2^-8 * 5 = 2.0e-2, typically by a few per cent
of that, and the result is rounded once more (2^-8 of |o|).  Bound used: 2e-2 max-abs, the bound of the
framework's attention, plus 2^-8 |o|.  log-sum-exp: scores are float32 sums (at most 128 * 2^-24 * sum|q k| scale
<= 1.8e-4 for these inputs, see below), the exponential and the sum add a few 2^-23; bound 3e-4 + 1e-6 |lse|.
float32: weights and outputs move by the scores' relative 1.8e-4 at most (worst case; sum|q k| scale < 2 sqrt(D));
bound 2e-4 * 5."""
import math

import numpy as np
import pytest

from oracle import ctcsd_oracle as orc
from paper_2412_00061_b200 import binding, synth


def _mask(rng, B, nodes, n_live):
    W = (nodes + 63) // 64
    m = np.zeros((B, nodes, W), dtype=np.uint64)
    for b in range(B):
        for i in range(n_live[b]):
            if i:
                m[b, i] = m[b, int(rng.integers(0, i))]
            m[b, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return m


def _inputs(rng, B, Hq, Hkv, D, dtype, nodes, n_live, pre, kv, Pcap=None, Lcap=None):
    n_live, pre, kv = (np.asarray(a, dtype=np.int32) for a in (n_live, pre, kv))
    Pcap = int(pre.max()) if Pcap is None else Pcap
    Lcap = int(max(1, (kv + n_live).max() + 3)) if Lcap is None else Lcap
    r = lambda *s: synth.to_dtype(np.clip(rng.normal(size=s), -5, 5).astype(np.float32), dtype)
    x = dict(Q=r(B, nodes, Hq, D), Kp=r(Hkv, Pcap, D), Vp=r(Hkv, Pcap, D), K=r(B, Hkv, Lcap, D), V=r(B, Hkv, Lcap, D),
             prefix_len=pre, kv_len=kv, n_nodes=n_live, mask=_mask(rng, B, nodes, n_live))
    return x


def _poison_hidden(x, value=np.nan):
    """Everything no row may look at: rows behind the lengths, queries of unused nodes."""
    for b in range(len(x["kv_len"])):
        end = x["kv_len"][b] + x["n_nodes"][b]
        x["K"][b, :, end:] = value
        x["V"][b, :, end:] = value
        x["Q"][b, x["n_nodes"][b]:] = value
    x["Kp"][:, x["prefix_len"].max():] = value
    x["Vp"][:, x["prefix_len"].max():] = value


class _Run:
    def __init__(self, x, dtype, with_lse=True):
        import torch
        self.t = torch
        B, nodes, Hq, D = x["Q"].shape
        Hkv = x["K"].shape[1]
        act = torch.bfloat16 if dtype == "bf16" else torch.float32
        d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
        self.h = binding.Handle(B, 64, 50, 5, 2, 8, 4, max(2, nodes), Hq, Hkv, D,
                                binding.DTYPE_BF16 if dtype == "bf16" else binding.DTYPE_F32)
        self.sa = self.h.make_shared_attention()
        self.d = {k: d(v).to(act) for k, v in x.items() if v.dtype == np.float32}
        self.d.update({k: d(v) for k, v in x.items() if v.dtype == np.int32})
        self.d["mask"] = d(x["mask"].view(np.int64))
        self.O = torch.full((B, nodes, Hq, D), 7.0, dtype=act, device="cuda:0")
        self.lse = torch.full((B, nodes, Hq), 7.0, device="cuda:0") if with_lse else None
        self.scale = 1.0 / math.sqrt(D)
        self.prefix = x["Kp"].shape[1] > 0

    def __call__(self):
        d = self.d
        kp, vp, pl = (d["Kp"], d["Vp"], d["prefix_len"]) if self.prefix else (None, None, None)
        self.h.tree_attention_shared(self.sa, d["Q"], kp, vp, pl, d["K"], d["V"], d["kv_len"], d["n_nodes"], d["mask"],
                                     self.scale, self.O, self.lse)
        return self

    def host(self):
        assert self.h.poll_status() == 0
        return self.O.float().cpu().numpy(), None if self.lse is None else self.lse.cpu().numpy()


def _oracle(x, scale):
    return orc.tree_attention_shared(x["Q"], x["Kp"], x["Vp"], x["prefix_len"], x["K"], x["V"], x["kv_len"], x["n_nodes"],
                                     x["mask"], scale)


def _check(O, lse, want_O, want_lse, dtype):
    tol = 2e-2 + 2.0 ** -8 * np.abs(want_O) if dtype == "bf16" else 1e-3
    assert np.all(np.isfinite(O) == np.isfinite(want_O))
    assert np.all(np.abs(O - want_O) <= tol), np.abs(O - want_O).max()
    if lse is not None:
        assert np.array_equal(np.isfinite(lse), np.isfinite(want_lse))
        assert np.all(lse[~np.isfinite(lse)] == -np.inf)
        f = np.isfinite(want_lse)
        err = np.abs(lse[f] - want_lse[f])
        assert np.all(err <= 3e-4 + 1e-6 * np.abs(want_lse[f])), err.max()


CASES = {   # B, Hq, Hkv, D, nodes, live nodes, prefix, cached
    "one_key": (1, 2, 2, 64, 2, [1], [0], [0]),
    "prefix_only": (2, 4, 2, 128, 4, [1, 1], [1, 1], [0, 0]),
    "no_prefix": (2, 4, 4, 128, 33, [33, 7], [0, 0], [5, 200]),
    "block_borders": (4, 4, 2, 128, 8, [8, 1, 3, 5], [128, 128, 128, 128], [128, 127, 124, 0]),
    "tokens": (9, 8, 8, 64, 2, [1] * 9, [300] * 9, [0, 1, 63, 64, 65, 127, 128, 129, 400]),
    "tokens_gqa": (40, 16, 2, 128, 2, [1] * 40, [200] * 40, [(37 * i) % 300 for i in range(40)]),
    "dead_between": (5, 8, 4, 128, 16, [0, 16, 0, 9, 0], [40] * 5, [10, 20, 30, 40, 50]),
    "all_dead": (2, 4, 2, 64, 8, [0, 0], [30, 30], [4, 4]),
    "spread": (6, 14, 2, 64, 21, [21, 3, 20, 11, 1, 8], [0, 500, 129, 128, 1, 77], [3, 0, 140, 260, 9, 64]),
    "trees": (3, 8, 2, 128, 64, [64, 40, 51], [640] * 3, [300, 129, 511]),
    "big_trees": (2, 8, 2, 128, 200, [200, 131], [257] * 2, [90, 33]),
    "odd_group": (3, 21, 3, 128, 40, [40, 39, 1], [333] * 3, [1, 2, 3]),
    "mqa": (2, 20, 1, 64, 30, [30, 29], [50, 20], [600, 0]),
    "many_tokens": (300, 4, 2, 64, 2, [(i * 7) % 3 for i in range(300)], [150] * 300, [(13 * i) % 40 for i in range(300)]),
    "many_spread": (1024, 2, 2, 64, 2, [1] * 1024, [(11 * i) % 130 for i in range(1024)], [i % 5 for i in range(1024)]),
    "long_split": (1, 4, 4, 128, 2, [2], [9001], [100]),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_shared_prefix_attention(name, dtype):
    B, Hq, Hkv, D, nodes, live, pre, kv = CASES[name]
    rng = np.random.default_rng([21, sorted(CASES).index(name)])
    x = _inputs(rng, B, Hq, Hkv, D, dtype, nodes, live, pre, kv, Pcap=max(pre) + (5 if max(pre) else 0))
    _poison_hidden(x)
    run = _Run(x, dtype)
    O, lse = run().host()
    want = _oracle(x, run.scale)
    _check(O, lse, *want, dtype)
    O2, lse2 = run().host()                      # the same workspace again
    assert np.array_equal(O, O2) and np.array_equal(lse, lse2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_what_the_mask_hides_does_not_reach_a_row(bad, dtype):
    """NaN and infinities in another branch of the tree, in another sequence's cache and in the part of the prefix
    that only others share: rows that do not see them are as the oracle has them without them."""
    rng = np.random.default_rng(22)
    B, Hq, Hkv, D, nodes = 4, 8, 4, 128, 24
    x = _inputs(rng, B, Hq, Hkv, D, dtype, nodes, [24, 10, 24, 5], [200, 90, 260, 260], [150, 30, 4, 77])
    clean = {k: v.copy() for k, v in x.items()}
    want_O, want_lse = _oracle(clean, 1.0 / math.sqrt(D))
    # sequence 2 goes bad as a whole; the prefix from row 230 on; node 3 of sequence 0
    x["K"][2], x["V"][2], x["Q"][2] = bad, bad, bad
    x["Kp"][:, 230:], x["Vp"][:, 230:] = bad, bad
    x["K"][0, :, 150 + 3], x["V"][0, :, 150 + 3] = bad, bad
    O, lse = _Run(x, dtype)().host()
    sees3 = [i for i in range(24) if (int(x["mask"][0, i, 0]) >> 3) & 1]
    ok0 = [i for i in range(24) if i not in sees3]
    assert sees3 and len(ok0) > 3
    _check(O[0, ok0], lse[0, ok0], want_O[0, ok0], want_lse[0, ok0], dtype)
    _check(O[1], lse[1], want_O[1], want_lse[1], dtype)
    if not np.isinf(bad) or bad > 0:             # (a key of -inf times a mixed-sign query is NaN as well)
        assert not np.any(np.isfinite(O[2]))
    if np.isnan(bad):
        assert np.all(np.isnan(O[0, sees3])) and np.all(np.isnan(O[3, :5]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_only_the_value_is_bad(dtype):
    """Finite keys, one NaN value: rows that see it are NaN, all others untouched (several splits of the keys)."""
    rng = np.random.default_rng(23)
    x = _inputs(rng, 3, 4, 2, 64, dtype, 8, [8, 8, 8], [700] * 3, [130, 260, 5])
    want = _oracle(x, 1.0 / 8.0)
    x["V"][1, :, 17] = np.nan
    O, lse = _Run(x, dtype)().host()
    assert np.all(np.isnan(O[1]))
    for b in (0, 2):
        _check(O[b], lse[b], want[0][b], want[1][b], dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_row_that_sees_nothing_is_zero(dtype):
    """Hand-made masks without the node's own bit, empty caches, no prefix."""
    rng = np.random.default_rng(24)
    x = _inputs(rng, 2, 4, 2, 64, dtype, 6, [6, 6], [0, 0], [0, 3])
    x["mask"][0, 2] = 0
    x["mask"][0, 5] = 1 << 1
    x["mask"][1, 4] = 0
    O, lse = _Run(x, dtype)().host()
    want = _oracle(x, 1.0 / 8.0)
    assert np.all(O[0, 2] == 0) and np.all(lse[0, 2] == -np.inf)
    _check(O, lse, *want, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scores_that_grow_from_block_to_block(dtype):
    """Every block moves the exponent's reference and rescales what has been accumulated; scores of hundreds."""
    rng = np.random.default_rng(25)
    x = _inputs(rng, 2, 8, 2, 128, dtype, 64, [64, 50], [1500, 1500], [700, 300])
    ramp = lambda n, s: (1.0 + 3.0 * ((np.arange(n) + s) // 128)).astype(np.float32)
    x["Kp"] = synth.to_dtype(x["Kp"] * ramp(x["Kp"].shape[1], 0)[None, :, None], dtype)
    x["K"] = synth.to_dtype(x["K"] * ramp(x["K"].shape[2], 1500)[None, None, :, None], dtype)
    run = _Run(x, dtype)
    O, lse = run().host()
    want_O, want_lse = _oracle(x, run.scale)
    # scores reach 55 * 5 times the usual ones: their float32 rounding (128 * 2^-24 * sum|q k| scale) grows alike, 1.8e-4 * 55
    assert np.abs(O - want_O).max() <= (2e-2 + 2.0 ** -8 * 5 if dtype == "bf16" else 5 * 1.8e-4 * 55)
    f = np.isfinite(want_lse)
    assert np.abs(lse[f] - want_lse[f]).max() <= 1.8e-4 * 55 + 1e-6 * np.abs(want_lse[f]).max()


@pytest.mark.gpu
def test_agrees_with_tree_attention_without_a_prefix():
    import torch
    rng = np.random.default_rng(26)
    x = _inputs(rng, 4, 16, 4, 128, "bf16", 64, [64, 33, 50, 1], [0] * 4, [400, 1, 129, 777])
    run = _Run(x, "bf16", with_lse=False)
    O, _ = run().host()
    d, out = run.d, torch.zeros_like(run.O)
    Lcap = max(x["K"].shape[2], 64)
    assert Lcap == x["K"].shape[2]
    run.h.tree_attention(d["Q"], d["K"], d["V"], d["kv_len"], d["n_nodes"], d["mask"], run.scale, out)
    assert run.h.poll_status() == 0
    assert np.abs(O - out.float().cpu().numpy()).max() <= 2e-2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bad_lengths_are_reported_and_the_others_served(dtype):
    rng = np.random.default_rng(27)
    x = _inputs(rng, 6, 4, 2, 64, dtype, 8, [8] * 6, [60] * 6, [40] * 6, Lcap=50)
    want = _oracle(x, 1.0 / 8.0)
    y = {k: v.copy() for k, v in x.items()}
    y["kv_len"][0], y["kv_len"][1] = 43, -1
    y["n_nodes"][2], y["n_nodes"][3] = 9, -2
    y["prefix_len"][4] = 61
    run = _Run(y, dtype)()
    assert run.h.poll_status() == -1 and run.h.poll_status() == 0
    O, lse = run.O.float().cpu().numpy(), run.lse.cpu().numpy()
    assert np.all(O[:5] == 0) and np.all(lse[:5] == -np.inf)
    _check(O[5:], lse[5:], want[0][5:], want[1][5:], dtype)


@pytest.mark.gpu
def test_refusals():
    import torch
    x = _inputs(np.random.default_rng(28), 2, 4, 2, 64, "bf16", 8, [8, 8], [60, 60], [40, 40])
    run = _Run(x, "bf16")
    d, h, sa = run.d, run.h, run.sa
    call = lambda scale=0.1, kp=d["Kp"], vp=d["Vp"], pl=d["prefix_len"], ws=sa, q=d["Q"]: h.tree_attention_shared(
        ws, q, kp, vp, pl, d["K"], d["V"], d["kv_len"], d["n_nodes"], d["mask"], scale, run.O, run.lse)
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(vp=None),
               dict(pl=None), dict(ws=dict(sa, ws_bytes=sa["ws_bytes"] - 1)), dict(q=d["Q"].float())):
        with pytest.raises(binding.CtcsdError):
            call(**kw)
    call()
    assert h.poll_status() == 0
    flat = torch.zeros(d["Q"].numel() + 1, dtype=torch.bfloat16, device="cuda:0")[1:].view(d["Q"].shape)    # 2-byte aligned
    with pytest.raises(binding.CtcsdError):
        call(q=flat)


def test_host_side_refusals_without_a_device():
    import ctypes
    lib = binding.load_library()
    n = ctypes.c_size_t(0)
    cfg = lambda B, nodes, Hq, Hkv, dt=1: binding.CConfig(B, 64, 50, 5, 2, 8, 4, nodes, Hq, Hkv, 64, dt, 0, 0)
    f = lib.ctcsd_tree_attention_shared_workspace_bytes
    assert f(ctypes.byref(cfg(2, 16, 4, 2)), ctypes.byref(n)) == 0 and n.value > 0
    assert f(ctypes.byref(cfg(1025, 16, 4, 2)), ctypes.byref(n)) == -2             # too many sequences
    assert f(ctypes.byref(cfg(1024, 256, 8, 2)), ctypes.byref(n)) == -2            # too many query rows
    assert f(ctypes.byref(cfg(2, 16, 4, 3)), ctypes.byref(n)) == -1 and f(None, ctypes.byref(n)) == -1
    assert lib.ctcsd_tree_attention_shared(None, None, None, 0, *([None] * 3), 0, *([None] * 3), 10, *([None] * 3), 1.0, None, None) == -1
