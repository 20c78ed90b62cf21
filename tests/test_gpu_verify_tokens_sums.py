"""Sums of a row that one lane adds up from more terms than 32 bits hold."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("V", [4095 * 512, 4200 * 512, 1 << 22])
def test_more_terms_than_a_32_bit_sum_holds(V):
    """With more requests than CTAs fit the GPU a request is one CTA of 512 threads, and a lane's share is V / 512 terms,
    every one of the largest weight. One row for all, by a stride of zero."""
    import paper_2401_14021_b200 as ralm
    R = 300
    target = torch.ones((1, 1, V), device=DEV).expand(R, 1, V)
    u = torch.arange(R, device=DEV, dtype=torch.float32)[:, None] / R
    u[R - 1] = 1.0 - 2.0 ** -24
    got, _ = ralm.verify_tokens(torch.empty((R, 0), dtype=torch.int64, device=DEV), None, target, u)
    # t = floor(V 2^40 U / 2^24) for U = floor(2^24 u), and token v is drawn for t in v 2^40 .. (v + 1) 2^40 - 1
    want = [(V << 40) * int(x * 2.0 ** 24) >> 24 >> 40 for x in u[:, 0].double().tolist()]
    assert got[:, 0].tolist() == want
