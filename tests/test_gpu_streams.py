"""The generator's calls on a stream that is not the current one, and inside a graph capture."""
import pytest
import torch

from test_gpu_kv_cache import DEV, attend_reference, check, filled, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def same_inputs_every_time():
    torch.manual_seed(0)


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


@pytest.mark.parametrize("given", ["neither", "k", "v"])
def test_results_of_a_read_on_another_stream(given):
    """Memory that queued work of the current stream still writes is not handed out for a result of another stream."""
    cache, k, v, b = filled(2, 2, 64, 16, [90, 40], seed=3)
    starts = i32([0, 0])
    want = [x.clone() for x in cache.read(0, starts, 90)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                  # loads the kernel, and leaves room in the other stream's allocator
        cache.read(0, starts, 90)
    own = torch.empty_like(want[0])
    torch.cuda.synchronize()
    blocks = [torch.empty_like(want[0]) for _ in range(4)]
    done = busy()
    for x in blocks:
        x.fill_(7.0)                               # comes after the wait
    del x, blocks                                  # free for the current stream to use again
    got = cache.read(0, starts, 90, k=own if given == "k" else None, v=own if given == "v" else None, stream=side)
    side.synchronize()
    assert not done.query()
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    assert got[0].dtype is torch.float16 and cache.device_status() == 0


def test_pages_and_tokens_on_another_stream():
    """Every call of the pages and the cache, in turn, on a stream that does not wait for the busy current one."""
    import paper_2401_14021_b200 as ralm
    x = torch.randn((3, 40, 2, 64), device=DEV).half()
    zero, lengths, grown = i32([0, 0, 0]), i32([40, 17, 0]), i32([40, 17, 43])
    new, starts, row = torch.randn((1, 3, 2, 64), device=DEV).half(), i32([40]), i32([2])
    src, dst = i32([0]), i32([2])
    out = torch.empty((3, 1, 4, 64), dtype=torch.float16, device=DEV)
    q = torch.randn((3, 1, 4, 64), device=DEV).half()
    k, v = (torch.empty((1, 43, 2, 64), dtype=torch.float16, device=DEV) for _ in range(2))

    def make():
        return ralm.KVCache.allocate(1, 2, 64, pages=12, rows=3, max_pages=4, page_size=16, device=DEV)

    def use(cache, stream):
        cache.resize(lengths, stream=stream)
        cache.append(0, x, x, zero, count=lengths, stream=stream)
        cache.fork(src, dst, stream=stream)
        cache.resize(grown, stream=stream)
        cache.append(0, new, new, starts, rows=row, stream=stream)
        cache.compact(stream=stream)
        cache.read(0, zero[:1], 43, rows=row, k=k, v=v, stream=stream)
        cache.attend(0, q, out=out, stream=stream)

    first, second = make(), make()
    use(first, None)
    want = [t.clone() for t in (first.table, first.lengths, first.refs, k, v, out)]
    for t in (k, v, out):
        t.zero_()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    done = busy()
    use(second, side)
    assert second.device_status(stream=side) == 0
    assert not done.query()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((second.table, second.lengths, second.refs, k, v, out), want))
    assert first.device_status() == 0
