"""The 4-bit operators where one kernel, pass or tile ends and the next begins, at the far end of a large cache, and from graphs that share a
workspace.  Cases, references and tolerances are those of the operators' own tests."""
import numpy as np
import pytest
import torch

import q4_util as u
import test_gpu_q4_attention as attention
import test_gpu_q4_draft as draft

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [7, 8, 16, 32, 33, 64, 65, 96, 97, 128, 129])
def test_draft_rows_at_the_edges_of_passes(M):
    c = draft._Case("bf16", M, 264, 300, 2, 3, 64, mapped=M % 2 == 1)
    c.run()
    c.check()


@pytest.mark.parametrize("H", [8, 120, 128, 136, 256, 264, 1032, 2048, 2056, 2184, 4104])
@pytest.mark.parametrize("M,group", [(1, 32), (40, 128)])
def test_draft_rows_of_odd_lengths(H, M, group):
    """One block, an odd number of them, a stretch of sums that ends with a block or two."""
    c = draft._Case("bf16", M, H, 2100, 3, 4, group)
    c.run()
    c.check()


@pytest.mark.parametrize("V,T", [(1, 1), (126, 8), (127, 8), (128, 5), (9472, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_draft_vocabularies_at_the_edges_of_tiles(dtype, V, T):
    c = draft._Case(dtype, 3, 384, V, T, 2 if V > 1 else 1, 32)
    c.run()
    c.check()


def test_draft_of_the_longest_float32_rows():
    c = draft._Case("fp32", 1, 44800, 20, 1, 2, 32)
    c.run()
    c.check()


def test_draft_of_bfloat16_rows_of_any_length():
    c = draft._Case("bf16", 2, 131072, 30, 1, 2, 128)
    c.run()
    c.check()


def test_classes_that_hold_no_number_leave_the_others_alone():
    rng = np.random.default_rng(4)
    w = rng.normal(size=(1, 200, 512)) * 0.05
    c = draft._Case("bf16", 4, 512, 199, 1, 3, 64, bias=False, weights=w)
    c.run()
    plain = c.z.clone()
    bad = torch.tensor([0, 31, 77, 198], device=u.DEV)
    c.W[0, bad, 100] = float("nan")
    c.Wq = c.h.quantize_weights_q4(c.W, 64)
    c.run()
    assert c.h.poll_status() == 0
    ok = torch.ones(200, dtype=torch.bool, device=u.DEV)
    ok[bad] = False
    assert torch.equal(c.z[..., ok], plain[..., ok]) and torch.isnan(c.z[..., bad]).all()


# rows of a kv head around the kernels' tiles (16, 128, 256), lengths around their blocks
@pytest.mark.parametrize("Hq,Hkv,nodes,n", [(1, 1, 16, 16), (1, 1, 17, 17), (1, 1, 128, 128), (1, 1, 129, 129), (2, 1, 8, 8), (2, 1, 9, 9),
                                            (4, 2, 128, 127), (4, 1, 64, 64), (4, 1, 65, 65)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_rows_and_lengths_at_the_edges_of_tiles(Hq, Hkv, nodes, n, D):
    kv = [0, 1, 127, 128, 191, 192, 193, 385]
    c = attention._Case("bf16", len(kv), Hq, Hkv, D, nodes, [n] * len(kv), kv, Lcap=393)
    c.run()
    c.check()


@pytest.mark.parametrize("nodes", [2, 20])
def test_attention_behind_2_to_the_32_bytes(nodes):
    """A cache whose levels take 4.4 GB a side: the last sequence's rows lie behind 2^32 bytes of levels and 2^33 values."""
    B, Hkv, D, Lcap, kv = 2, 8, 128, 4_300_000, 300
    c = attention._Case("bf16", B, Hkv, Hkv, D, nodes, [nodes, nodes], [0, kv])
    h = c.h
    big = h.make_q4_cache(Lcap)
    for name in ("Kq", "Vq", "Ks", "Vs"):
        assert big[name].numel() * big[name].element_size() > (2 ** 32 if name[1] == "q" else 2 ** 29)
        small = c.cache[name]
        big[name][:, :, :small.shape[2]] = small
    c.run()
    want = c.O.clone(), c.lse.clone()
    c.cache = big
    c.run()
    c.check()
    assert torch.equal(c.O, want[0]) and torch.equal(c.lse, want[1])


def test_two_graphs_of_one_workspace_replayed_in_turn():
    a = attention._Case("bf16", 2, 8, 2, 128, 40, [40, 21], [1000, 333], seed=1)
    b = attention._Case("bf16", 2, 8, 2, 128, 40, [3, 40], [77, 2000], seed=2)
    for c in (a, b):
        c.run()
        c.check()
    b.h, b.ws = a.h, a.ws
    want = [(c.O.clone(), c.lse.clone()) for c in (a, b)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    for c in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.run()
        graphs.append(g)
    for _ in range(3):
        for c in (a, b):
            c.O.zero_()
            c.lse.zero_()
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for c, w in zip((a, b), want):
        assert torch.equal(c.O, w[0]) and torch.equal(c.lse, w[1])


def test_rows_stored_on_another_stream_are_read_behind_it():
    c = attention._Case("bf16", 3, 4, 4, 64, 6, [6, 2, 1], [300, 41, 5])
    c.run()
    want = c.O.clone()
    for name in ("Kq", "Vq", "Ks", "Vs"):
        c.cache[name].zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.h.store_rows_q4(c.cache, c.K, c.V, u.i32([c.K.shape[2]] * 3), stream=s)
    c.run(stream=s)
    s.synchronize()
    assert c.h.poll_status() == 0 and torch.equal(c.O, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,V", [(1, 8), (3, 300), (20, 32), (40, 129)])
def test_a_blank_that_is_ruled_out(dtype, M, V):
    """blank_bias = -inf: the blank has no part in the sum and ranks last."""
    c = draft._Case(dtype, M, 256, V, 2, 3, 32)
    c.bias.fill_(-np.inf)
    c.run()
    assert c.h.poll_status() == 0
    z, tol = c.reference()
    assert torch.all(z[..., V] == -np.inf) and torch.all(c.z[..., V] == -np.inf)
    ids = c.z.sort(dim=-1, descending=True, stable=True)[1]
    assert torch.equal(c.out[0].long(), ids[..., :3])
    assert torch.all((c.out[2].double() - torch.logsumexp(z, -1)).abs() <= tol[..., :V].amax(-1) + 3e-5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hq,nodes", [(2, 3), (2, 40), (2, 200)])
def test_a_batch_without_nodes_and_one_without_rows(dtype, Hq, nodes):
    for n, kv in (([0, 0, 0], [50, 0, 7]), ([0, nodes, 1], [0, 0, 0])):
        c = attention._Case(dtype, 3, Hq, 1, 64, nodes, n, kv)
        c.run()
        c.check()


def test_a_cache_whose_tensors_are_exchanged_is_checked_again():
    c = attention._Case("bf16", 1, 2, 1, 64, 3, [3], [70])
    c.run()
    want = c.O.clone()
    good = dict(c.cache)
    c.cache |= {name: t.clone() for name, t in good.items()}
    for t in good.values():
        t.zero_()
    c.run()
    assert torch.equal(c.O, want)
    c.cache["Vs"] = c.cache["Vs"][:, :, :5].contiguous()
    with pytest.raises(u.binding.CtcsdError):
        c.run()
    short = c.h.make_q4_cache(20)
    short["Kq"].resize_(1, 1, 10, 32)
    with pytest.raises(u.binding.CtcsdError):
        c.h.store_rows_q4(short, c.K, c.V, u.i32([10]))
