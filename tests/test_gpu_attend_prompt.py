"""Attention of whole prompts over the 4-bit cache: tens to hundreds of queries per entry, many blocks of query rows, with
and without tokens before them. Tolerance as in test_gpu_kv_cache.py."""
import pytest
import torch

from test_gpu_kv_cache import DEV, attend_reference, check, filled, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def same_inputs_every_time():
    torch.manual_seed(0)


@pytest.mark.parametrize("D,ps", [(64, 16), (128, 64)])
@pytest.mark.parametrize("n,H,G,lengths", [(10, 2, 1, [10]), (33, 1, 1, [33, 40]), (33, 2, 3, [33, 5, 300]), (128, 1, 4, [128, 161]),
                                           (130, 2, 1, [130, 131, 700]), (509, 1, 4, [509, 1000])])
def test_prompts_match_definition(D, ps, n, H, G, lengths):
    cache, k, v, b = filled(len(lengths), H, D, ps, lengths, seed=n)
    q = (1.5 * torch.randn((len(lengths), n, H * G, D), device=DEV)).half()
    got = cache.attend(0, q)
    assert cache.device_status() == 0
    check(got, *attend_reference(q, k, v, b, lengths, D ** -0.5))


def test_prompts_of_different_lengths_in_one_call():
    """q_len from nothing to all of n, rows in another order, bf16."""
    lengths = [200, 64, 130, 77]
    cache, k, v, b = filled(4, 2, 64, 32, lengths, seed=3)
    rows, q_len = [2, 0, 3, 1], [130, 0, 77, 33]
    q = torch.randn((4, 130, 6, 64), device=DEV).bfloat16()
    got = cache.attend(0, q, rows=i32(rows), q_len=i32(q_len))
    assert cache.device_status() == 0
    check(got, *attend_reference(q, k[rows], v[rows], b[rows], [lengths[r] for r in rows], 0.125, q_len))
