"""Attention over rows and values whose sizes differ by more than a 16-bit number spans. Tolerance as in test_gpu_kv_cache.py."""
import pytest
import torch

from test_gpu_kv_cache import DEV, attend_reference, check, give_pages, i32, make_cache, stands_for

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def same_inputs_every_time():
    torch.manual_seed(0)


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


# ---- weights of very different sizes
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,G", [(1, 1), (1, 8), (2, 8), (3, 8), (4, 8)])
@pytest.mark.parametrize("gap", [6.0, 9.0, 12.0, 16.0])
def test_small_weights_count_where_the_largest_stands_for_nothing(D, n, G, gap):
    """Where the token with nearly all the weight stands for exactly 0, the others are the result, though their weights are
    exp(-gap) of its."""
    cache, order = make_cache(1, 1, D, 16, 4, seed=4)
    give_pages(cache, order, [48 + n])
    g = torch.Generator(DEV).manual_seed(int(gap))
    k = torch.randn((1, 48 + n, 1, D), generator=g, device=DEV)
    k = 0.5 * (k - k.mean(-1, keepdim=True))                     # scores of 0
    v = 0.2 * torch.randn((1, 48 + n, 1, D), generator=g, device=DEV)
    k[0, 21] = 1.0                                               # a score of gap
    v[0, 21], v[0, 21, 0, 0], v[0, 21, 0, 1] = 0.0, -2.0, 1.75   # steps of 0.25, no offset
    k, v = k.half(), v.half()
    cache.append(0, k, v, i32([0]))
    (dk, _), (dv, bv) = values_of(k), values_of(v)
    assert (dv[0, 21, 0, 2:] == 0).all() and (bv[0, 21] == 0).all()
    q = torch.ones((1, n, G, D), device=DEV).half()
    check(cache.attend(0, q, scale=gap / D), *attend_reference(q, dk, dv, bv, [48 + n], gap / D))


# ---- values of very different sizes
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,G", [(1, 2), (3, 4), (5, 4), (8, 4)])
@pytest.mark.parametrize("length,at,gap", [(300, 0, 3), (300, 70, -4), (300, 64, 25), (300, 280, 3), (300, 40, 150), (7000, 3333, -2),
                                           (7000, 3300, 20)])
@pytest.mark.parametrize("size", [1e-1, 1e-3, 1e-4])
def test_a_large_value_that_does_not_count_costs_the_others_nothing(D, n, G, length, at, gap, size):
    """One token's values are the largest that the format holds. For half of the query rows its weight is exp(-40) of that of
    the token `gap` positions on, which counts most; for the others it is nearly all."""
    cache, order = make_cache(1, 1, D, 64, -(-length // 64), seed=2)
    give_pages(cache, order, [length])
    g = torch.Generator(DEV).manual_seed(at)
    k = 0.3 * torch.randn((1, length, 1, D), generator=g, device=DEV)
    v = size * torch.randn((1, length, 1, D), generator=g, device=DEV)
    k[0, at + gap] = 1.5
    k[0, at] = -6.0
    v[0, at] = 57344.0 * (2.0 * torch.rand((1, D), generator=g, device=DEV) - 1.0)
    k, v = k.half(), v.half()
    cache.append(0, k, v, i32([0]))
    (dk, _), (dv, bv) = values_of(k), values_of(v)
    q = torch.ones((1, n, G, D), device=DEV).half()
    q[0, :, 1::2] = -1.0                                         # these rows see the large value and little else
    for scale in (8.0 / D, 4.0 / D):
        got = cache.attend(0, q, scale=scale)
        assert cache.device_status() == 0
        check(got, *attend_reference(q, dk, dv, bv, [length], scale))


# ---- the weight that counts most is exact
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [1.0, 0.013, 3e-5, 9000.0])
def test_a_row_of_one_token_is_that_tokens_value(dtype, D, size):
    """Its p is a power of two but for the rounding of the score less its reference (2^-20 where scores stay below 8), so
    p s_v becomes a power of two times s_v in fp16, which is exact: s (c - 8) loses nothing to the weight's 11 bits. What
    remains is 2^-19 of |v| + |b|, and the result's half unit."""
    B, H, G = 40, 2, 4
    cache, order = make_cache(B, H, D, 16, 1, seed=5)
    give_pages(cache, order, [1] * B)
    g = torch.Generator(DEV).manual_seed(5)
    k = torch.randn((B, 1, H, D), generator=g, device=DEV).half()
    v = (size * (torch.randn((B, 1, H, D), generator=g, device=DEV) + 0.3)).half()
    cache.append(0, k, v, i32([0] * B))
    want, offset = (x.repeat_interleave(G, 2) for x in values_of(v))
    q = torch.randn((B, 1, H * G, D), generator=g, device=DEV).to(dtype)
    got = cache.attend(0, q).double()
    info = torch.finfo(dtype)
    unit = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=info.tiny)))) * info.eps
    assert ((got - want).abs() <= 0.5 * unit + 2.0 ** -19 * (want.abs() + offset.abs())).all()
