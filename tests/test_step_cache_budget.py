"""The step's cache budget on the CPU: what DraftVerifyStep itself does around the calls.  The library's handle is replaced
by a stand-in whose calls change the same buffers in a way that is easy to follow (every step accepts one draft token, the
gathered weight of a cached row is how often it was looked at, an eviction fills row 0 from the first row behind the budget),
so that no test here needs a GPU."""
import numpy as np
import pytest
import torch

from paper_2412_00061_b200 import binding, synth
from paper_2412_00061_b200.step import DraftVerifyStep

CFG = synth.CONFIGS["c1"].replace(name="stand_in", B=2, H=8, V=20, Hq=2, Hkv=2, D=4, kv_lo=4, kv_hi=9, max_nodes=3, T=2)
LCAP = 24


class _Handle:
    """Stands in for binding.Handle."""

    def __init__(self, *args, **kw):
        self.calls = []

    def __getattr__(self, name):                       # any other call: noted, changes nothing
        if name.startswith("_"):
            raise AttributeError(name)
        return lambda *a, **kw: self.calls.append(name)

    def make_shared_attention(self):
        return dict(ws=torch.zeros(1))

    def make_eviction(self, Lcap):
        return dict(Lcap=Lcap)

    def poll_status(self):
        return 0

    def build_tree(self, base_tok, kv_len, cand_tok, cand_len, n_cand, node_tok, parent, depth, pos, *rest, stream=None):
        self.calls.append("build_tree")
        pos.copy_(kv_len[:, None].expand_as(pos))

    def tree_attention_shared(self, ws, Q, Kp, Vp, prefix_len, K, V, kv_len, n_nodes, mask, scale, out_O, out_lse=None, stream=None):
        self.calls.append("tree_attention_shared")
        for b in range(K.shape[0]):
            out_O[b] = K[b, :, :int(kv_len[b])].double().sum().float()

    def commit_accepted(self, K, V, kv_len, acc_len, acc_nodes, out_kv_len, out_sel_row, stream=None):
        self.calls.append("commit_accepted")
        out_kv_len.copy_(kv_len + 2)

    def attention_mass(self, Q, K, kv_len, acc_len, acc_nodes, lse, scale, mass, row_pos, n_evicted=None, decay=1.0, stream=None):
        self.calls.append("attention_mass")
        for b in range(K.shape[0]):
            n = int(kv_len[b])
            mass[b, :, :n] = mass[b, :, :n] * decay + 1.0
            row_pos[b, :, n - 2:n] = torch.arange(n - 2, n, dtype=torch.int32) + n_evicted[b]

    def evict_rows(self, ev, K, V, mass, row_pos, kv_len, n_evicted, budget, sinks, recent, out_mass, out_row_pos, out_kv_len,
                   out_n_evicted, stream=None):
        self.calls.append("evict_rows")
        for b in range(K.shape[0]):
            n = int(kv_len[b])
            if n > budget:
                for t in (K, V, mass, row_pos):
                    t[b, :, 0] = t[b, :, budget]
                kv_len[b] = budget
                n_evicted[b] += n - budget


@pytest.fixture()
def step(monkeypatch):
    monkeypatch.setattr(binding, "Handle", _Handle)
    s = DraftVerifyStep(CFG, device="cpu")
    g = torch.Generator().manual_seed(3)
    r = lambda *shape: torch.randn(*shape, generator=g)
    s.set_inputs(K=r(CFG.B, CFG.Hkv, LCAP, CFG.D), V=r(CFG.B, CFG.Hkv, LCAP, CFG.D), Wd=None, Wl=None,
                 kv_len=torch.tensor([4, 9], dtype=torch.int32), base_tok=torch.zeros(CFG.B, dtype=torch.int32))
    return s


def _chain(s, n_steps=5):
    g = torch.Generator().manual_seed(5)
    r = lambda *shape: torch.randn(*shape, generator=g)
    n = CFG.max_nodes
    s.setup_chain(n_steps, r(CFG.B, CFG.H), torch.zeros(CFG.B, dtype=torch.int32), torch.tensor([4, 9], dtype=torch.int32),
                  r(n_steps, CFG.B, n, CFG.Hq, CFG.D), r(n_steps, CFG.B, CFG.Hkv, n, CFG.D), r(n_steps, CFG.B, CFG.Hkv, n, CFG.D),
                  r(n_steps, CFG.B * n, CFG.H))


def _state(s):
    k = s.cache
    return [t.clone() for t in (s.inp["K"], s.inp["V"], k["mass"], k["row_pos"], k["n_evicted"], s.chain["kv_len"])]


@pytest.mark.parametrize("budget_first", [True, False])
def test_a_chain_with_a_budget_runs_again_from_its_start(step, budget_first):
    K0, V0 = step.inp["K"].clone(), step.inp["V"].clone()
    if budget_first:
        step.enable_cache_budget(8, sinks=1, recent=2, decay=0.5, Lcap=LCAP)
    _chain(step)
    if not budget_first:
        step.enable_cache_budget(8, sinks=1, recent=2, decay=0.5, Lcap=LCAP)
    # by hand: two tokens a step from 4 and 9 cached rows, cut to 8
    kv, ev, base = np.array([4, 9]), np.array([0, 0]), []
    for _ in range(5):
        base.append(kv + ev)
        ev = ev + np.maximum(kv + 2 - 8, 0)
        kv = np.minimum(kv + 2, 8)
    runs = []
    for _ in range(3):
        step.run_chain()
        runs.append(_state(step) + [step.chain["rec"][k].clone() for k in ("pos", "O", "new_kv_len")])
        np.testing.assert_array_equal(step.chain["rec"]["pos"][:, :, 0].numpy(), np.stack(base))
        np.testing.assert_array_equal(step.cache["n_evicted"].numpy(), ev)
        # the first step looked at the start's rows
        want = [K0[b, :, :n].double().sum().float() for b, n in enumerate((4, 9))]
        assert [step.chain["rec"]["O"][0][b, 0, 0, 0].item() for b in range(2)] == [w.item() for w in want]
    for r in runs[1:]:
        for a, b in zip(r, runs[0]):
            assert torch.equal(a, b)
    assert not torch.equal(step.inp["K"], K0) and not torch.equal(step.inp["V"], V0)


def test_a_new_batch_in_the_same_buffers_starts_afresh(step):
    """reset_cache() and other rows in K and V: as a step that never saw the first batch."""
    step.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    _chain(step)
    step.run_chain()
    tensors = [step.cache[k] for k in ("mass", "row_pos", "n_evicted")]
    g = torch.Generator().manual_seed(9)
    K1, V1 = (torch.randn(step.inp["K"].shape, generator=g) for _ in range(2))
    step.inp["K"].copy_(K1)
    step.inp["V"].copy_(V1)
    step.reset_cache()
    assert all(a is b for a, b in zip(tensors, [step.cache[k] for k in ("mass", "row_pos", "n_evicted")]))      # in place
    assert step.cache["mass"].abs().max() == 0 and step.cache["n_evicted"].abs().max() == 0
    assert torch.equal(step.cache["row_pos"], torch.arange(LCAP, dtype=torch.int32).expand_as(step.cache["row_pos"]))
    step.run_chain()
    got = _state(step)
    step.run_chain()
    for a, b in zip(_state(step), got):
        assert torch.equal(a, b)

    other = DraftVerifyStep(CFG, device="cpu")
    other.set_inputs(K=K1.clone(), V=V1.clone(), Wd=None, Wl=None, base_tok=step.inp["base_tok"])
    other.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    _chain(other)
    other.run_chain()
    for a, b in zip(got, _state(other)):
        assert torch.equal(a, b)


def test_other_buffers_begin_a_chain_of_their_own(step):
    """K and V replaced through set_inputs(): the old rows do not come back into the new buffers."""
    step.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    _chain(step)
    step.run_chain()
    K1, V1 = torch.ones_like(step.inp["K"]), torch.ones_like(step.inp["V"])
    step.set_inputs(K=K1, V=V1)
    step.reset_cache()
    step.run_chain()
    assert step.chain["rec"]["O"][0][1, 0, 0, 0].item() == 9 * CFG.Hkv * CFG.D


def test_one_sequence_is_replaced(step):
    step.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    _chain(step)
    step.run_chain()
    before = {k: step.cache[k].clone() for k in ("mass", "row_pos", "n_evicted")}
    step.reset_cache([1])
    k = step.cache
    assert k["mass"][1].abs().max() == 0 and k["n_evicted"][1] == 0
    assert torch.equal(k["row_pos"][1], torch.arange(LCAP, dtype=torch.int32).expand_as(k["row_pos"][1]))
    assert all(torch.equal(k[n][0], before[n][0]) for n in before)
    for bad in ([2], [-1]):
        with pytest.raises(ValueError):
            step.reset_cache(bad)


def test_enabling_the_budget_again_keeps_its_tensors(step):
    """What a captured graph points at stays in use; its contents start afresh."""
    step.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    tensors = [step.cache[k] for k in ("mass", "row_pos", "n_evicted")]
    for t in tensors:
        t.fill_(7)
    step.enable_cache_budget(10, sinks=1, recent=2, decay=0.5, Lcap=LCAP)
    assert all(a is b for a, b in zip(tensors, [step.cache[k] for k in ("mass", "row_pos", "n_evicted")]))
    assert step.cache["mass"].abs().max() == 0 and step.cache["n_evicted"].abs().max() == 0
    assert (step.cache["budget"], step.cache["decay"]) == (10, 0.5)


def test_reset_without_a_budget_is_refused(step):
    with pytest.raises(ValueError):
        step.reset_cache()


@pytest.mark.parametrize("kw", [dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(sinks=5, recent=4), dict(decay=1.5), dict(decay=-0.1),
                                dict(decay=float("nan")), dict(Lcap=LCAP + 1), dict(budget=LCAP), dict(budget=16, sinks=4, recent=64)])
def test_limits_that_no_commit_would_take_are_refused_at_once(step, kw):
    """The library refuses these too, but only inside the first commit, behind the history update.  A refusal leaves a
    budget that was set before as it is."""
    args = dict(dict(budget=8, sinks=1, recent=2, decay=0.5, Lcap=LCAP), **kw)
    with pytest.raises(ValueError):
        step.enable_cache_budget(**args)
    assert step.cache is None and step.shared is None
    step.enable_cache_budget(8, sinks=1, recent=2, decay=0.5, Lcap=LCAP)
    before = dict(step.cache)
    with pytest.raises(ValueError):
        step.enable_cache_budget(**args)
    assert step.cache == before


def test_the_caches_rows_are_taken_from_them(step):
    step.enable_cache_budget(8, sinks=1, recent=2)
    assert step.cache["Lcap"] == LCAP and step.cache["mass"].shape[2] == LCAP


@pytest.mark.parametrize("name", ["K", "V"])
def test_caches_of_another_size_are_refused(step, name):
    step.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    before = dict(step.inp)
    with pytest.raises(ValueError):
        step.set_inputs(**{name: torch.zeros(CFG.B, CFG.Hkv, LCAP + 2, CFG.D), "kv_len": None})
    assert all(step.inp[k] is before[k] for k in before)


def test_the_same_buffers_given_again_are_no_new_batch(step):
    """set_inputs() with the tensors that are in use already, between two runs of a chain."""
    step.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    _chain(step)
    step.run_chain()
    got = _state(step)
    step.set_inputs(K=step.inp["K"], V=step.inp["V"])
    step.run_chain()
    for a, b in zip(_state(step), got):
        assert torch.equal(a, b)


def test_another_budget_for_the_same_chain(step):
    """enable_cache_budget() between two runs: the chain still begins at its own start, with nothing dropped."""
    K0, V0 = step.inp["K"].clone(), step.inp["V"].clone()
    step.enable_cache_budget(8, sinks=1, recent=2, Lcap=LCAP)
    _chain(step)
    step.run_chain()
    step.enable_cache_budget(6, sinks=1, recent=2, decay=0.5, Lcap=LCAP)
    step.run_chain()

    other = DraftVerifyStep(CFG, device="cpu")
    other.set_inputs(K=K0, V=V0, Wd=None, Wl=None, base_tok=step.inp["base_tok"])
    other.enable_cache_budget(6, sinks=1, recent=2, decay=0.5, Lcap=LCAP)
    _chain(other)
    other.run_chain()
    for a, b in zip(_state(step), _state(other)):
        assert torch.equal(a, b)
