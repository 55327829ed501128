"""The cache operators under the debug-bounds build (the indices of their stores into the callers' arrays, workspaces, plans and lists are
checked; a failed check is recorded in the status word and the store is skipped): the tests of the regular build, each of which asserts a clean
status word and the oracle's results."""
import pytest

import test_gpu_cache_ops as ops
import test_gpu_evict_moves as moves
import test_gpu_mass_blocks as blocks
import test_gpu_shared_attention as shared
import test_gpu_shared_attention_mix as mix

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def debug_library():
    from paper_2412_00061_b200 import binding, build
    lib = binding.use_library(build.build(debug_bounds=True))
    assert lib.ctcsd_debug_bounds_enabled() == 1
    yield lib
    assert binding.use_library(None).ctcsd_debug_bounds_enabled() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", ["one_key", "no_prefix", "block_borders", "dead_between", "all_dead", "spread", "big_trees", "mqa",
                                  "many_tokens", "many_spread", "long_split"])
def test_shared_attention(name, dtype):
    shared.test_shared_prefix_attention(name, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("seed", range(4))
def test_shared_attention_of_drawn_shapes(seed, dtype):
    mix.test_drawn_shapes(seed, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", sorted(ops.MASS))
def test_mass(name, dtype):
    ops.test_gathered_weight(name, dtype)


@pytest.mark.parametrize("name", ["two_tiles", "tensor_memory", "two_passes", "fp32_two_chunks"])
def test_mass_of_many_blocks(name):
    blocks.test_many_blocks_and_pieces_per_cta(name, 64)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", sorted(ops.EVICT))
def test_eviction(name, in_place, dtype):
    ops.test_eviction(name, True, dtype, in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_eviction_of_many_pairs(in_place):
    moves.test_lists_of_moves_at_the_limit_of_shared_memory(in_place)
