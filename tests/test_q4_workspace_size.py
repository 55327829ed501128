"""The 4-bit draft head works in scratch that a handle has anyway: a handle's workspace is as large as before there were 4 bits."""
import ctypes

import pytest

from paper_2412_00061_b200 import binding, synth

# bytes of a handle's workspace without the 4-bit operators
FORMER = {"c1": 1650432, "c2": 1650432, "c3": 5850112, "c4": 6898688, "c5": 70372352, "c6": 3749888}


def _bytes(**kw):
    c = dict(B=1, H=4096, V=32000, T=5, k=4, beam=0, topN=16, max_nodes=64, Hq=32, Hkv=32, D=128, dtype=1, score_mode=0, max_draft_rows=0)
    c.update(kw)
    n = ctypes.c_size_t(0)
    assert binding.load_library().ctcsd_workspace_bytes(ctypes.byref(binding.CConfig(*c.values())), ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("name", sorted(FORMER))
def test_the_configurations(name):
    c = synth.CONFIGS[name]
    assert _bytes(B=c.B, H=c.H, V=c.V, T=c.T, k=c.k, beam=c.beam, topN=c.topN, max_nodes=c.max_nodes, Hq=c.Hq, Hkv=c.Hkv, D=c.D,
                  dtype=1 if c.dtype == "bf16" else 0, score_mode=c.score_mode) == FORMER[name]


@pytest.mark.parametrize("rows,former", [(32, 30936832), (128, 30936832)])
def test_many_draft_rows_of_an_ordinary_vocabulary(rows, former):
    assert _bytes(max_draft_rows=rows) == former


@pytest.mark.parametrize("B,H", [(1, 8), (1, 131072), (4, 8192), (8, 8192)])
def test_few_rows_of_a_small_vocabulary(B, H):
    assert _bytes(B=B, H=H, V=30, T=1, max_nodes=8) == _bytes(B=B, H=H, V=30, T=1, max_nodes=8, dtype=0)


def test_many_rows_of_a_small_vocabulary_take_what_they_need():
    """Where the other draft heads need less: rows of a pass (128 at most), and a state for each, four times for 160 SMs and two slots."""
    for rows in (16, 100, 128, 1000):
        most = min(rows, 128)
        assert _bytes(max_draft_rows=rows, V=30, T=1, max_nodes=8) <= 1650432 + most * 4096 * 2 + 80 * 4 * most * 160 * 2 + 80 * 4 * (rows + 127) // 128 * 128 + 512
