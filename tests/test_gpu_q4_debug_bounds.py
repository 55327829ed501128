"""The 4-bit operators under the debug-bounds build (the indices of their stores into the callers' arrays and the workspaces are checked; a failed check
is recorded in the status word and the store is skipped): tests of the regular build, each of which asserts a clean status word and the results."""
import pytest

import test_gpu_q4_attention as attention
import test_gpu_q4_chain as chain
import test_gpu_q4_edges as edges
import test_gpu_q4_rows as rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def debug_library():
    from paper_2412_00061_b200 import binding, build
    lib = binding.use_library(build.build(debug_bounds=True))
    assert lib.ctcsd_debug_bounds_enabled() == 1
    yield lib
    assert binding.use_library(None).ctcsd_debug_bounds_enabled() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", attention.SHAPES)
def test_attention(dtype, shape):
    attention.test_outputs_and_lse(dtype, *shape)


@pytest.mark.parametrize("rows_of", [(1, 1, 17, 17), (1, 1, 129, 129), (4, 1, 65, 65)])
def test_attention_at_the_edges_of_tiles(rows_of):
    edges.test_attention_rows_and_lengths_at_the_edges_of_tiles(*rows_of, 64)


@pytest.mark.parametrize("dtype,B,Hkv,D", rows.SHAPES)
def test_rows(dtype, B, Hkv, D):
    rows.test_store_then_load(dtype, B, Hkv, D, 33)
    rows.test_commit(dtype, B, Hkv, D, True)


def test_sequences_that_leave_their_arrays():
    rows.test_sequences_that_leave_their_arrays_are_left_unchanged()


@pytest.mark.parametrize("M", [8, 33, 129])
def test_draft(M):
    edges.test_draft_rows_at_the_edges_of_passes(M)


@pytest.mark.parametrize("layout", ["packed", "raw"])
def test_chain(layout):
    chain.test_chained_steps_in_4_bits("mha", layout)
