"""The draft heads over 16-bit and 4-bit weights of one handle share its scratch: called in turn, and replayed in turn, each gives what it
gives alone."""
import pytest
import torch

import test_gpu_q4_draft as draft
import q4_util as u

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,H,V", [(1, 4096, 3000), (4, 1024, 500), (8, 512, 4000), (20, 512, 4000), (33, 264, 50), (130, 72, 400)])
def test_both_heads_in_turn(M, H, V):
    c = draft._Case("bf16", M, H, V, 2, 3, 64, mapped=True)
    other = [torch.zeros_like(t) for t in c.out]
    c.run(dbg=False)
    want = [t.clone() for t in c.out]
    x = c.x[c.x_rows.long()].contiguous()
    plain = lambda: c.h.draft_logits(x, c.W, c.row_seq, c.bias, *other)
    plain()
    want_other = [t.clone() for t in other]
    c.run()
    c.check()

    def clear():
        for t in c.out + other:
            t.zero_()

    def check():
        torch.cuda.synchronize()
        assert c.h.poll_status() == 0
        assert all(torch.equal(a, b) for a, b in zip(c.out, want)) and all(torch.equal(a, b) for a, b in zip(other, want_other))

    for _ in range(5):
        clear()
        for _ in range(3):
            plain()
            c.run(dbg=False)
        check()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        for _ in range(2):
            c.run(dbg=False)
            plain()
    clear()
    g.replay()
    check()


@pytest.mark.parametrize("dtype,M,H,V,T,k,group", [("bf16", 8, 2048, 500, 2, 8, 64), ("bf16", 17, 4096, 130, 2, 4, 128), ("bf16", 130, 72, 400, 2, 4, 32),
                                                   ("fp32", 1, 8, 3, 1, 1, 32), ("fp32", 9, 520, 47, 8, 8, 128), ("fp32", 4, 1000, 9000, 3, 2, 32)])
def test_the_4_bit_head_under_the_debug_bounds_build(dtype, M, H, V, T, k, group):
    """Every index of a store that is formed from data lies in its array (the status word stays clean)."""
    from paper_2412_00061_b200 import binding, build
    assert binding.use_library(build.build(debug_bounds=True)).ctcsd_debug_bounds_enabled() == 1
    try:
        c = draft._Case(dtype, M, H, V, T, k, group, mapped=True)
        c.run()
        c.check()
    finally:
        binding.use_library(None)
