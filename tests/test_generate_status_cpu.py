"""Which device and stream the status of a pool is read on: host logic, with a CUDA of two devices played by fakes."""
import contextlib

import pytest
import torch


class FakeCuda:
    """torch.cuda's current device and streams; what is asked for is on record."""

    def __init__(self, monkeypatch):
        self.now, self.log = 0, []
        for name in ("device", "stream", "current_stream"):
            monkeypatch.setattr(torch.cuda, name, getattr(self, name))
        self.streams = {d: FakeStream(100 + d) for d in range(2)}

    @contextlib.contextmanager
    def device(self, d):
        before, self.now = self.now, torch.device(d).index
        yield
        self.now = before

    @contextlib.contextmanager
    def stream(self, s):
        before = self.streams[self.now]
        if s is not None:
            self.streams[self.now] = s
        yield
        self.streams[self.now] = before

    def current_stream(self, device=None):
        return self.streams[self.now if device is None else torch.device(device).index]


class FakeStream:
    def __init__(self, number):
        self.cuda_stream = number


class FakeTensor:
    def __init__(self, cuda, device):
        self.cuda, self.device = cuda, torch.device("cuda", device)

    def zero_(self):
        self.cuda.log.append(("zero", self.cuda.now, self.cuda.current_stream().cuda_stream))


class FakeLibrary:
    def __init__(self, cuda, status):
        self.cuda, self.status = cuda, status

    def ralm_pages_status(self, pages, stream):
        self.cuda.log.append(("status", self.cuda.now, stream))
        return self.status


@pytest.fixture
def cuda(monkeypatch):
    return FakeCuda(monkeypatch)


def pool(cls, cuda, device, status):
    cache = object.__new__(cls)
    cache.table, cache._lib, cache._ptr = FakeTensor(cuda, device), FakeLibrary(cuda, status), 0
    cache._attend_work = FakeTensor(cuda, device)
    return cache


@pytest.mark.parametrize("device", [0, 1])
def test_status_is_read_on_the_pools_device(cuda, device):
    from paper_2401_14021_b200 import KVCache, Pages
    for cls in (Pages, KVCache):
        cuda.log.clear()
        assert pool(cls, cuda, device, 1).device_status() == 1
        assert pool(cls, cuda, device, 0).device_status(stream=FakeStream(7)) == 0
        assert cuda.log == [("status", device, 100 + device), ("status", device, 7)] and cuda.now == 0


@pytest.mark.parametrize("device", [0, 1])
def test_the_workspace_is_cleared_on_the_same_stream_after_a_timeout(cuda, device):
    from paper_2401_14021_b200 import KVCache
    assert pool(KVCache, cuda, device, 4).device_status() == 4
    assert pool(KVCache, cuda, device, 4).device_status(stream=FakeStream(7)) == 4
    assert cuda.log == [("status", device, 100 + device), ("zero", device, 100 + device), ("status", device, 7), ("zero", device, 7)]
