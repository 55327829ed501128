"""The index checks of the debug-bounds build in the 4-bit operators: where they stand (read from the sources)."""
import pytest

from test_debug_bounds_sites import _sites


@pytest.mark.parametrize("kernel_file,stores", [
    ("draft_q4.cuh", 2),                   # log-sum-exp, the k best
    ("draft_logits_q4.cu", 5),             # packing: levels, scales and origins; float32: logits, warps' states, the CTA's state
    ("draft_logits_q4_tc.cu", 4),          # warps' states, logits, the CTA's state, gathered rows
    ("rows_q4.cu", 3),                     # storing, reading back, history update
    ("q4_attention.cuh", 3),               # rows of unused nodes, their log-sum-exp, the cuts
    ("tree_attention_q4.cu", 3), ("tree_attention_q4_mma.cu", 2), ("tree_attention_q4_tc.cu", 4),
])
def test_the_4_bit_operators_check_what_they_store(kernel_file, stores):
    assert len(_sites()[kernel_file]) >= stores

