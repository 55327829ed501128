"""Shared-prefix attention refuses capacities whose key blocks it could not number, before anything is launched (the bound
itself is tested on the host: shared_plan_host.cu)."""
import ctypes

import pytest

from paper_2412_00061_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [binding.DTYPE_BF16, binding.DTYPE_F32])
@pytest.mark.parametrize("Pcap,Lcap", [(2147483000, 512), (0, 2147483000)])
def test_capacities_past_the_plans_numbers(Pcap, Lcap, dtype):
    import torch
    B, nodes, Hq, Hkv, D = 64, 256, 4, 2, 64
    h = binding.Handle(B, 64, 50, 5, 2, 8, 4, nodes, Hq, Hkv, D, dtype)
    sa = h.make_shared_attention()
    small = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda:0")       # (looked at by no kernel: refused)
    p, before = small.data_ptr(), h.launch_count
    rc = h.lib.ctcsd_tree_attention_shared(h._h, None, sa["ws_ptr"], sa["ws_bytes"], p, p, p, Pcap, p, p, p, Lcap, p, p, p,
                                           ctypes.c_float(0.125), p, p)
    assert rc == -2 and h.launch_count == before
