"""A 4-bit cache's tensors are looked at by every call, whatever they were at the call before: on the CPU, with the device check of
the binding's pointers left out."""
import pytest
import torch

from paper_2412_00061_b200 import binding

B, HKV, LCAP, D = 2, 3, 10, 64


@pytest.fixture()
def handle(monkeypatch):
    ptr = binding._ptr

    class _OnDevice:                             # a CPU tensor that says it is on the device
        def __init__(self, t):
            self.t = t

        def __getattr__(self, name):
            return True if name == "is_cuda" else getattr(self.t, name)

    monkeypatch.setattr(binding, "_ptr", lambda t, *a: ptr(None if t is None else _OnDevice(t), *a))
    h = binding.Handle.__new__(binding.Handle)
    h.cfg, h.device, h._h = binding.CConfig(B=B, Hkv=HKV, D=D), torch.device("cpu"), None
    return h


def test_a_cache_is_known_by_its_four_tensors(handle):
    cache = handle.make_q4_cache(LCAP)
    ptrs, rows = handle._q4_cache(cache)
    assert rows == LCAP and list(ptrs) == [cache[k].data_ptr() for k in ("Kq", "Ks", "Vq", "Vs")]
    assert list(handle._q4_cache(dict(cache))[0]) == list(ptrs)


@pytest.mark.parametrize("name", ["Kq", "Ks", "Vq", "Vs"])
@pytest.mark.parametrize("seen", [False, True])
def test_a_tensor_that_is_changed_in_place_is_refused(handle, name, seen):
    """The tensor stays the same object at the same address; its sizes, strides or type do not."""
    for change in (lambda t: t.resize_(B, HKV, LCAP - 1, t.shape[3]) if t.dim() == 4 else t.resize_(B, HKV, LCAP - 1, *t.shape[3:]),
                   lambda t: t.transpose_(1, 2)):
        cache = handle.make_q4_cache(LCAP)
        if seen:
            handle._q4_cache(cache)
        at = cache[name].data_ptr()
        change(cache[name])
        assert cache[name].data_ptr() == at
        with pytest.raises(binding.CtcsdError):
            handle._q4_cache(cache)


def test_a_cache_that_is_resized_as_a_whole_has_its_new_rows(handle):
    cache = handle.make_q4_cache(LCAP)
    handle._q4_cache(cache)
    for k in cache:
        cache[k].resize_(B, HKV, LCAP - 3, *cache[k].shape[3:])
    assert handle._q4_cache(cache)[1] == LCAP - 3
