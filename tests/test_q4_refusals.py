"""What the 4-bit calls refuse on the host, without a device: sizes, groups, null pointers (status codes of the C entries)."""
import ctypes

import pytest

from paper_2412_00061_b200 import binding


def _cfg(**kw):
    c = dict(B=1, H=4096, V=32000, T=5, k=4, beam=0, topN=16, max_nodes=64, Hq=32, Hkv=32, D=128, dtype=1, score_mode=0, max_draft_rows=0)
    c.update(kw)
    return binding.CConfig(*c.values())


def test_sizes_of_packed_weights():
    lib = binding.load_library()
    n = ctypes.c_size_t(0)
    for group, block in ((32, 1280), (64, 1152), (128, 1088)):
        assert lib.ctcsd_weights_q4_bytes(ctypes.byref(_cfg()), group, ctypes.byref(n)) == 0
        assert n.value == 5 * 2001 * 32 * block
    assert lib.ctcsd_weights_q4_bytes(ctypes.byref(_cfg(H=136, V=15)), 128, ctypes.byref(n)) == 0
    assert n.value == 5 * 1 * 2 * 1088
    for group in (0, -32, 16, 96, 256):
        assert lib.ctcsd_weights_q4_bytes(ctypes.byref(_cfg()), group, ctypes.byref(n)) == -1
    assert lib.ctcsd_weights_q4_bytes(None, 128, ctypes.byref(n)) == -1
    assert lib.ctcsd_weights_q4_bytes(ctypes.byref(_cfg()), 128, None) == -1
    assert lib.ctcsd_weights_q4_bytes(ctypes.byref(_cfg(D=96)), 128, ctypes.byref(n)) == -1


def test_workspace_of_the_attention():
    lib = binding.load_library()
    n = ctypes.c_size_t(0)
    assert lib.ctcsd_tree_attention_q4_workspace_bytes(ctypes.byref(_cfg()), ctypes.byref(n)) == 0
    assert 0 < n.value < (1 << 28)
    assert lib.ctcsd_tree_attention_q4_workspace_bytes(ctypes.byref(_cfg(B=1025, max_nodes=2)), ctypes.byref(n)) == -2
    assert lib.ctcsd_tree_attention_q4_workspace_bytes(ctypes.byref(_cfg(max_nodes=1)), ctypes.byref(n)) == -1
    assert lib.ctcsd_tree_attention_q4_workspace_bytes(None, ctypes.byref(n)) == -1


@pytest.mark.parametrize("name", ["quantize_weights_q4", "draft_logits_q4", "store_rows_q4", "load_rows_q4", "commit_accepted_q4", "tree_attention_q4"])
def test_a_call_without_a_handle_is_refused(name):
    fn = getattr(binding.load_library(), "ctcsd_" + name)
    ptrs = [1 if t in (ctypes.c_int, ctypes.c_size_t) else (1.0 if t is ctypes.c_float else None) for t in fn.argtypes]
    assert fn(*ptrs) == -1
