"""Which workspace binding.KvCache gives a call, with torch replaced: no GPU is used."""
import contextlib
from types import SimpleNamespace

import pytest

from paper_2507_04453_b200 import binding


class FakeTorch:
    """Two devices, each with a current stream that is being captured or not."""

    uint8 = "uint8"

    def __init__(self, current=0):
        self.current, self.capturing = current, {0: False, 1: False}
        self.cuda = SimpleNamespace(current_device=lambda: self.current, is_current_stream_capturing=lambda: self.capturing[self.current],
                                    device=self._on, stream=lambda s: self._on(s.device_index))

    @contextlib.contextmanager
    def _on(self, index):
        before, self.current = self.current, index
        try:
            yield
        finally:
            self.current = before

    def empty(self, n, dtype, device):
        return SimpleNamespace(shape=(n,), device=device)


def cache_on(torch, index):
    kv = binding.KvCache.__new__(binding.KvCache)
    kv.ctx, kv.device, kv._index, kv._ws = SimpleNamespace(torch=torch), f"cuda:{index}", index, {}
    return kv


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("stream", [None, SimpleNamespace(device_index=1)])
def test_a_captured_call_has_a_workspace_of_its_own_whatever_device_is_current(current, stream):
    torch = FakeTorch(current)
    kv = cache_on(torch, 1)
    eager = kv._workspace(100, 7, stream)
    assert kv._workspace(100, 7, stream) is eager and kv._workspace(60, 7, stream) is eager  # a stream's calls take turns
    assert kv._workspace(100, 8, stream) is not eager
    torch.capturing[1] = True
    a, b = kv._workspace(100, 7, stream), kv._workspace(100, 7, stream)
    assert a is not eager and b is not eager and a is not b
    torch.capturing[1] = False
    assert kv._workspace(100, 7, stream) is eager
    torch.capturing[0] = True  # a capture on the other device is not this cache's
    assert kv._workspace(100, 7, stream) is eager and torch.current == current


def test_a_workspace_that_is_too_small_is_replaced():
    kv = cache_on(FakeTorch(), 0)
    first = kv._workspace(100, None, None)
    second = kv._workspace(101, None, None)
    assert second is not first and second.shape[0] == 101 and kv._workspace(100, None, None) is second
