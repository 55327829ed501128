"""The index checks of the debug-bounds build: where they stand (read from the sources)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_00061_b200", "csrc")


def _sites():
    found = {}
    for f in sorted(os.listdir(CSRC)):
        if f == "common.cuh":
            continue
        with open(os.path.join(CSRC, f)) as src:
            found[f] = [int(m) for m in re.findall(r"CTCSD_IN_BOUNDS\([^,]+, (\d+),", src.read())]
    return found


@pytest.mark.parametrize("kernel_file,stores", [
    ("tree_attention_shared.cu", 4),       # plain kernel: outputs, parts; merge: unused rows, outputs
    ("tree_attention_shared_tc.cu", 4),    # parts (output, reference and sum), outputs, log-sum-exp
    ("shared_attention.cuh", 3),           # the plan, the published plan
    ("attention_mass.cu", 1), ("attention_mass.cuh", 1),
    ("evict_rows.cu", 6),                  # lists, kept rows, moved rows, their weights
])
def test_the_cache_operators_check_what_they_store(kernel_file, stores):
    assert len(_sites()[kernel_file]) >= stores


def test_a_site_number_names_one_file():
    at = {}
    for f, numbers in _sites().items():
        for n in set(numbers):
            assert n not in at, "site %d stands in %s and in %s" % (n, at[n], f)
            at[n] = f
