"""Packing weights on a stream of one's own: what orders it against the current stream, and keeps the allocator from handing memory on too early.
On the CPU, with stand-ins that note what is done: the order is what the test is about."""
import types

import pytest
import torch

from paper_2412_00061_b200 import binding


class _Stream:
    def __init__(self, name, log):
        self.name, self.log, self.cuda_stream = name, log, 7 if name == "current" else 8

    def wait_stream(self, other):
        self.log.append(("wait", self.name, other.name))


class _Tensor:
    """Stands in for a CUDA tensor."""

    def __init__(self, name, log):
        self.name, self.log = name, log

    def record_stream(self, s):
        self.log.append(("record", self.name, s.name))


@pytest.fixture()
def packing(monkeypatch):
    log = []
    current = _Stream("current", log)

    class _Lib:
        def ctcsd_weights_q4_bytes(self, cfg, group, out):
            return 0

        def ctcsd_quantize_weights_q4(self, *a):
            log.append(("pack",))
            return 0

    h = binding.Handle.__new__(binding.Handle)
    h.lib, h._h, h._dev, h.device, h.act_dtype, h.cfg = _Lib(), None, 0, torch.device("cpu"), torch.float32, binding.CConfig()

    def empty(*a, **kw):
        log.append(("allocate", "w"))
        return _Tensor("w", log)

    monkeypatch.setattr(binding, "torch", types.SimpleNamespace(
        empty=empty, uint8=torch.uint8, cuda=types.SimpleNamespace(current_stream=lambda device=None: current, Stream=_Stream)))
    monkeypatch.setattr(binding, "_ptr", lambda t, *a: 1)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream, device=None: 7)
    return h, log, current


def test_a_side_stream_waits_and_holds_what_it_reads_and_writes(packing):
    h, log, current = packing
    side = _Stream("side", log)
    h.quantize_weights_q4(_Tensor("Wd", log), 64, stream=side)
    at = {e: i for i, e in enumerate(log)}
    # the packed weights' memory may still be in use by what was queued on the current stream: packing waits for it
    assert at[("allocate", "w")] < at[("wait", "side", "current")] < at[("pack",)]
    # both are in use on the side stream when the caller lets go of them
    assert ("record", "w", "side") in at and ("record", "Wd", "side") in at


def test_packing_in_place_waits_and_holds_too(packing):
    h, log, current = packing
    h.quantize_weights_q4(_Tensor("Wd", log), 64, stream=_Stream("side", log), out=dict(w=_Tensor("old", log), group=64))
    assert log.index(("wait", "side", "current")) < log.index(("pack",))
    assert ("record", "old", "side") in log and ("record", "Wd", "side") in log


@pytest.mark.parametrize("given", [False, True])
def test_nothing_of_that_on_the_current_stream(packing, given):
    h, log, current = packing
    h.quantize_weights_q4(_Tensor("Wd", log), 64, stream=_Stream("current", log) if given else None)
    assert not any(e[0] == "wait" for e in log) and ("pack",) in log
