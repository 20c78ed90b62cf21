"""Attention over rows and values whose sizes differ by more than a 16-bit number spans. Tolerance as in test_gpu_kv_cache.py."""
import pytest
import torch

from test_gpu_kv_cache import DEV, attend_reference, check, give_pages, i32, make_cache, stands_for

pytestmark = pytest.mark.gpu


def values_of(x):
    held, _, offset = stands_for(x)
    return torch.from_numpy(held).to(DEV), torch.from_numpy(offset).to(DEV)


# ---- query rows of very different sizes
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,G", [(1, 1), (1, 8), (2, 8), (3, 8), (4, 8), (9, 4)])
@pytest.mark.parametrize("factor", [1e4, 1e9, 1e20, 1e30])
def test_a_row_does_not_depend_on_its_neighbours_size(D, n, G, factor):
    lengths = [90, 400]
    cache, order = make_cache(2, 2, D, 32, 13, seed=1)
    give_pages(cache, order, lengths)
    g = torch.Generator(DEV).manual_seed(int(n + G))
    k, v = (torch.randn((2, 400, 2, D), generator=g, device=DEV).half() for _ in range(2))
    cache.append(0, k, v, i32([0, 0]), count=i32(lengths))
    (dk, _), (dv, bv) = values_of(k), values_of(v)
    q = torch.randn((2, n, 2 * G, D), generator=g, device=DEV)
    small = q.bfloat16()
    want, size = attend_reference(small, dk, dv, bv, lengths, D ** -0.5)
    alone = cache.attend(0, small)
    check(alone, want, size)
    for big in {0, 2 * G - 1}:
        mixed = q.clone()
        mixed[:, n // 2, big] *= factor
        got = cache.attend(0, mixed.bfloat16())
        assert got.isfinite().all()
        keep = torch.ones((n, 2 * G), dtype=torch.bool, device=DEV)
        keep[n // 2, big] = False
        check(got[:, keep], want[:, keep], size[:, keep])
    # and rows that are all small or all large, the scale making up for it
    for x in (factor, 1.0 / factor):
        scaled = (q * x).bfloat16()
        s = D ** -0.5 / x
        check(cache.attend(0, scaled, scale=s), *attend_reference(scaled, dk, dv, bv, lengths, s))
