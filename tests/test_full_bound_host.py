"""The bound that a full-context cache keeps on the host of how many slots are in use, without a GPU: the library's calls and torch's queries of the
current device and capture are stood in for."""
import types

import pytest
import torch

from paper_2505_23666_amd import binding as lb


@pytest.fixture
def cache(monkeypatch):
    """A cache on device 1 while device 0 is the current one; device 1's current stream is being captured where `capturing` says so."""
    world = types.SimpleNamespace(device=0, capturing=False, calls=[])

    class on:
        def __init__(self, device):
            self.device = device.index

        def __enter__(self):
            self.was, world.device = world.device, self.device

        def __exit__(self, *_):
            world.device = self.was

    monkeypatch.setattr(torch.cuda, "current_device", lambda: world.device)
    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: world.capturing and world.device == 1)
    for name in ("lola_full_init", "lola_full_evict", "lola_full_append"):
        monkeypatch.setattr(lb, name, lambda *a, n=name: world.calls.append((n, world.device)))
    c = lb.LolaFullCache.__new__(lb.LolaFullCache)
    c.device, c.capacity, c.cfg, c.st, c.fill, c._captured = torch.device("cuda:1"), 128, None, None, 100, False
    c.count = torch.full((1, 1), 100, dtype=torch.int32)
    c._ws = lambda T, gather: None
    c.world = world
    return c


@pytest.mark.parametrize("call", ["evict", "reset"])
def test_a_captured_call_does_not_lower_the_bound(cache, call):
    """What is only recorded has not happened: the bound stays, and later calls look at the counts."""
    cache.world.capturing = True
    cache.evict(10) if call == "evict" else cache.reset()
    assert cache.world.calls == [("lola_full_" + ("evict" if call == "evict" else "init"), 1)]
    assert cache.fill == 100 and cache._captured
    cache.world.capturing = False
    with pytest.raises(lb.LolaError, match="evict first"):
        cache._on_device(cache._append, None, None, None, 40)


@pytest.mark.parametrize("call", ["evict", "reset"])
def test_a_call_outside_a_capture_lowers_it(cache, call):
    cache.evict(10) if call == "evict" else cache.reset()
    assert cache.fill == (10 if call == "evict" else 0) and not cache._captured
    cache._on_device(cache._append, None, None, None, 40)
    assert cache.fill == (50 if call == "evict" else 40)
