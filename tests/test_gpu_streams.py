"""The generator's calls on a stream that is not the current one, and inside a graph capture."""
import pytest
import torch

from test_gpu_kv_cache import DEV, attend_reference, check, filled, i32

pytestmark = pytest.mark.gpu


def busy(milliseconds=60):
    """Keeps the current stream busy; the event that is returned comes after that."""
    torch.cuda._sleep(int(milliseconds * 1.9e6))
    done = torch.cuda.Event()
    done.record()
    return done


def dirty(bytes_):
    """Leaves the current stream's allocator with blocks that hold anything but zeros."""
    blocks = [torch.full((bytes_,), 0x55, dtype=torch.uint8, device=DEV) for _ in range(3)]
    torch.cuda.synchronize()
    del blocks


@pytest.mark.parametrize("n,G", [(1, 1), (3, 4), (9, 4)])
def test_first_attention_on_another_stream(n, G):
    """Rows that are split over many CTAs, whose counters have to be clear before the first call of these sizes."""
    lengths = [9000, 100, 2500]
    dirty(64 << 20)
    cache, k, v, b = filled(3, 2, 64, 16, lengths, seed=1)
    q = torch.randn((3, n, 2 * G, 64), device=DEV).half()
    want, size = attend_reference(q, k, v, b, lengths, 0.125)
    side = torch.cuda.Stream()
    # what may wait for the device by itself comes first: loading a kernel, memory for another stream
    filled(3, 2, 64, 16, lengths, seed=1)[0].attend(0, q)
    outs = [torch.zeros_like(q) for _ in range(3)]
    torch.cuda.synchronize()
    done = busy()
    got = [cache.attend(0, q, out=out, stream=side) for out in outs]
    side.synchronize()
    assert not done.query()                        # the current stream has not come to anything yet
    kept = [x.cpu() for x in got]
    torch.cuda.synchronize()
    for x in kept:
        check(x.to(DEV), want, size)
    assert cache.device_status() == 0
    check(cache.attend(0, q), want, size)          # and nothing came late


def test_first_attention_inside_a_capture():
    lengths = [5000, 70]
    dirty(64 << 20)
    cache, k, v, b = filled(2, 2, 64, 16, lengths, seed=2)
    q = torch.randn((2, 2, 4, 64), device=DEV).half()
    want, size = attend_reference(q, k, v, b, lengths, 0.125)
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cache.attend(0, q, out=out)
    check(cache.attend(0, q), want, size)          # before the graph has run once
    graph.replay()
    check(out, want, size)
    check(cache.attend(0, q), want, size)
    assert cache.device_status() == 0
