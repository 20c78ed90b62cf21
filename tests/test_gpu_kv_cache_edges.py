"""The 4-bit cache at its edges: entries without tokens, positions outside a row."""
import pytest
import torch

from test_gpu_kv_cache import DEV, give_pages, i32, make_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def same_inputs_every_time():
    torch.manual_seed(0)


# ---- entries without tokens, positions outside a row
@pytest.mark.parametrize("D", [64, 128])
def test_an_entry_without_tokens_is_no_error(D):
    cache, order = make_cache(3, 2, D, 16, 4)
    give_pages(cache, order, [18, 16, 0])
    x = torch.randn((3, 5, 2, D), device=DEV).half()
    cache.fork(i32([0]), i32([2]))                            # rows 0 and 2 share their pages
    before = cache.pool.clone()
    for starts in ([18, 16, 18], [18, 18, 17], [5, 30, 0], [63, 64, 200]):
        cache.append(0, x, x, i32(starts), count=i32([0, 0, 0]))
        assert cache.device_status() == 0
        cache.append(0, x, x, i32(starts), count=i32([-3, 0, -1]))
        assert cache.device_status() == 0
    assert torch.equal(cache.pool, before)
    cache.resize(i32([18, 20, 18]))                            # one entry of three has tokens
    cache.append(0, x, x, i32([18, 18, 18]), count=i32([0, 2, 0]))
    assert cache.device_status() == 0
    back, _ = cache.read(0, i32([18]), 2, rows=i32([1]))
    assert (back != 0).any()


@pytest.mark.parametrize("D", [64, 128])
def test_reading_outside_a_row_gives_zeros_and_no_error(D):
    cache, order = make_cache(2, 2, D, 16, 4)
    give_pages(cache, order, [16, 0])
    x = torch.randn((1, 16, 2, D), device=DEV).half()
    cache.append(0, x, x, i32([0]), rows=i32([0]))
    for start, rows in ((18, [0]), (31, [0]), (3, [1]), (60, [1]), (-40, [0]), (-3, [1]), (2 ** 31 - 20, [0]), (-2 ** 31, [0])):
        k, v = cache.read(0, i32([start]), 7, rows=i32(rows))
        assert (k == 0).all() and (v == 0).all() and cache.device_status() == 0, start


def test_tokens_outside_a_row_are_reported():
    cache, order = make_cache(1, 1, 64, 16, 4)
    give_pages(cache, order, [20])
    x = torch.randn((1, 6, 1, 64), device=DEV).half()
    before = cache.pool.clone()
    for start in (20, 25, 33, 64, 2 ** 31 - 7, -6, -7, -30, -2 ** 31):
        cache.append(0, x, x, i32([start]))
        assert cache.device_status() == 1, start
    assert torch.equal(cache.pool, before)
