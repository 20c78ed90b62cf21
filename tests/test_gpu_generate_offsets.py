"""Strides that take offsets beyond 2^31 elements and 2^32 bytes, in every tensor that may be strided: the results are those of
dense copies, bit for bit where the alignment is the same."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FAR = 2 ** 31 + 8                                   # elements


@pytest.fixture(scope="module")
def room():
    buffer = torch.zeros(4 * (FAR + 4096), dtype=torch.uint8, device=DEV)        # 8.6 GB
    yield buffer
    del buffer
    torch.cuda.empty_cache()


def far(room, x, dim):
    """A copy of x whose `dim`, of size 2, has a stride of FAR elements."""
    strides, at = [0] * x.dim(), 1
    for d in reversed(range(x.dim())):
        strides[d] = at
        at *= x.shape[d] if d != dim else 1
    strides[dim] = FAR
    assert at <= 4096
    y = room.view(x.dtype).as_strided(x.shape, strides)
    y.copy_(x)
    return y


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_mixture(room, dtype):
    import paper_2401_14021_b200 as ralm
    torch.manual_seed(0)
    x = torch.randn((2, 1000), device=DEV).to(dtype)
    want = ralm.knn_mix(x, None, None, None, 0.5)
    assert torch.equal(ralm.knn_mix(far(room, x, 0), None, None, None, 0.5), want)
    out = far(room, torch.zeros((2, 1000), device=DEV), 0)
    assert torch.equal(ralm.knn_mix(x, None, None, None, 0.5, probs=out), want)


@pytest.mark.parametrize("dim", [0, 1])
def test_verification(room, dim):
    import paper_2401_14021_b200 as ralm
    torch.manual_seed(0)
    R, S, V = (2, 1, 300) if dim == 0 else (3, 1, 300)
    target = torch.softmax(torch.randn((R, S + 1, V), device=DEV), -1)
    draft = torch.softmax(torch.randn((R, S + (dim == 1), V), device=DEV), -1)
    tokens = torch.randint(0, V, (R, S), device=DEV)
    u = torch.rand((R, S + 1), device=DEV)
    want = ralm.verify_tokens(tokens, draft[:, :S], target, u)
    got = ralm.verify_tokens(tokens, draft[:, :S], far(room, target, dim), u)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = ralm.verify_tokens(tokens, far(room, draft, dim)[:, :S], target, u)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dim", [0, 1, 2])
def test_cache(room, dim):
    import paper_2401_14021_b200 as ralm
    torch.manual_seed(0)
    cache = ralm.KVCache.allocate(1, 2, 64, pages=8, rows=2, max_pages=4, page_size=16, device=DEV)
    lengths, zero = torch.tensor([20, 7], dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    cache.resize(lengths)
    k, v = (torch.randn((2, 2, 2, 64), device=DEV).half() for _ in range(2))
    x = torch.randn((2, 20, 2, 64), device=DEV).half()
    cache.append(0, x, x, zero, count=lengths)
    cache.append(0, k, v, zero)
    want = cache.read(0, zero, 2)
    cache.append(0, v, k, zero)                     # something else in between
    cache.append(0, far(room, k, dim), v, zero)
    assert all(torch.equal(a, b) for a, b in zip(cache.read(0, zero, 2), want))
    cache.append(0, v, k, zero)
    cache.append(0, k, far(room, v, dim), zero)
    assert all(torch.equal(a, b) for a, b in zip(cache.read(0, zero, 2), want))
    assert torch.equal(cache.read(0, zero, 2, k=far(room, torch.zeros_like(k), dim))[0], want[0])
    assert torch.equal(cache.read(0, zero, 2, v=far(room, torch.zeros_like(k), dim), k=torch.empty_like(k))[1], want[1])
    q = torch.randn((2, 2, 2, 64), device=DEV).half()
    out = cache.attend(0, q)
    assert torch.equal(cache.attend(0, far(room, q, dim)), out)
    assert torch.equal(cache.attend(0, q, out=far(room, torch.zeros_like(q), dim)), out)
    assert cache.device_status() == 0
