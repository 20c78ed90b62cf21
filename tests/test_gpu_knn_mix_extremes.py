"""The KNN-LM mixture where exponents are large: masks of any size, temperatures of any size, scores of any size.

Tolerance, set from the arithmetic. The kernel scales by fl(log2(e) / T), which is within 2^-23 of its value and the same
factor everywhere, so an exponent's difference from the row's largest, d, is off by 2^-23 |d| for the factor, 2^-24 |d| each
for the difference and the product. Where the result is above 2^-100 of the row's largest that is 100 * 2^-22 * ln 2 = 1.7e-5
relative; the approximate 2^x, the sums and the division add a few 2^-22. So 2e-5 relative, and 1e-30 for what is smaller."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ralm():
    import paper_2401_14021_b200 as ralm
    return ralm


def reference(logits, ids, scores, values, lam, T, tau, sign):
    """The definition in 64 bits; every row has a logit above -inf and no NaN."""
    lm = torch.softmax(logits.double().cpu() / T, 1)
    if ids is None:
        return lm
    out = (1.0 - lam) * lm
    for r in range(logits.shape[0]):
        w = torch.softmax(sign * scores[r].double().cpu() / tau, 0)
        out[r].index_put_((values[ids[r]].long().cpu(),), lam * w, accumulate=True)
    return out


def check(got, want):
    got = got.double().cpu()
    assert got.isfinite().all()
    assert ((got - want).abs() <= 2e-5 * want + 1e-30).all(), ((got - want).abs() / (want + 1e-30)).max()


def neighbours(R, V, k, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    values = torch.randint(0, V, (500,), generator=g, device=DEV, dtype=torch.int32)
    return torch.randint(0, 500, (R, k), generator=g, device=DEV), 40.0 * torch.rand((R, k), generator=g, device=DEV), values


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [37, 32000])
def test_rows_masked_with_any_constant(dtype, V):
    """Every logit the same, whatever it is: uniform."""
    ralm = _ralm()
    levels = [-1e4, -1e6, -3e6, -1e7, -1e9, -1e10, -1e12, -1e15, -1e18, -3e38, 1e6, 1e9, 1e12, 1e17, 3e38]
    logits = torch.tensor(levels, device=DEV)[:, None].expand(-1, V).to(dtype).contiguous()
    ids, scores, values = neighbours(len(levels), V, 6, 1)
    for T in (1.0, 0.8, 1e3):
        check(ralm.knn_mix(logits, None, None, None, 0.5, temperature=T), reference(logits, None, None, None, 0.5, T, 1.0, -1))
        check(ralm.knn_mix(logits, ids, scores, values, 0.3, temperature=T, knn_temperature=7.0),
              reference(logits, ids, scores, values, 0.3, T, 7.0, -1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [53, 32000])
def test_some_logits_masked_with_any_constant(dtype, V):
    ralm = _ralm()
    g = torch.Generator(DEV).manual_seed(2)
    levels = [-1e4, -1e9, -1e10, -1e12, -3e38]
    logits = (3.0 * torch.randn((len(levels), V), generator=g, device=DEV)).to(dtype)
    for r, x in enumerate(levels):
        logits[r, V // 3:] = x
    check(ralm.knn_mix(logits, None, None, None, 0.5), reference(logits, None, None, None, 0.5, 1.0, 1.0, -1))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1e-4, 1e-6, 1e-8, 1e-9, 1e-20, 1e-37, 1e6, 1e30, 3e38])
def test_temperatures_of_any_size(dtype, T):
    """Towards 0 the largest logit takes all (ties share), towards infinity the row is uniform."""
    ralm = _ralm()
    g = torch.Generator(DEV).manual_seed(3)
    for V, top in ((200, 20.0), (32000, 20.0), (200, -5.0)):
        logits = (top + torch.randn((3, V), generator=g, device=DEV)).to(dtype)
        logits[2, :] = logits[2, :].abs().neg()
        logits[2, V // 2] = 0.0
        check(ralm.knn_mix(logits, None, None, None, 0.5, temperature=T), reference(logits, None, None, None, 0.5, T, 1.0, -1))


def test_parts_of_a_row_around_the_change_of_form():
    """Exponents around 2^22, where the kernel goes from one form of its powers to the other: parts of a row below,
    above and across it, in the CTAs of a cluster and the warps of a CTA."""
    ralm = _ralm()
    V = 32000
    g = torch.Generator(DEV).manual_seed(4)
    for sign in (1.0, -1.0):
        edge = sign * 2.0 ** 22 / math.log2(math.e)              # 2907270: a step of fp32 is 0.25
        for low, high in ((-8, -1), (1, 8), (-6, 6)):
            other = torch.randint(-32, 32, (2, V), generator=g, device=DEV) / 4.0
            logits = (edge + other).float()
            part = torch.randint(4 * low, 4 * high, (2, V), generator=g, device=DEV) / 4.0
            logits[0, : V // 2] = (edge + part[0, : V // 2]).float()
            logits[1, 4000:4300] = (edge + part[1, 4000:4300]).float()
            logits[1, 4300:] = (edge - 20.0 - other[1, 4300:].abs()).float()
            check(ralm.knn_mix(logits, None, None, None, 0.5), reference(logits, None, None, None, 0.5, 1.0, 1.0, -1))


def test_scores_of_any_size():
    """Finite scores count, whatever they are and whatever the temperature makes of them; the tolerance holds for scores that
    are large beside their differences too, as only the differences are scaled."""
    ralm = _ralm()
    R, V, k = 6, 97, 24
    g = torch.Generator(DEV).manual_seed(5)
    logits = torch.randn((R, V), generator=g, device=DEV)
    ids, _, values = neighbours(R, V, k, 6)
    near = 10.0 * torch.rand((R, k), generator=g, device=DEV)
    for metric, sign in ((ralm.IP, 1), (ralm.L2, -1)):
        for scores, tau in ((near + 1e4, 1.0), (near.round() + 1e6, 2.0), (near + 3e4, 10.0), (near - 2e4, 1.0),
                            (torch.full_like(near, 1e30), 1e-10), (torch.full_like(near, -3e38), 1e-3), (near * 1e37, 1e-5),
                            ((near - 5.0) * 6e37, 1.0), (near, 1e-37), (near, 3e38), (near * 1e37, 3e38)):
            got = ralm.knn_mix(logits, ids, scores, values, 0.6, knn_temperature=tau, metric=metric)
            check(got, reference(logits, ids, scores, values, 0.6, 1.0, tau, sign))


def test_scores_whose_difference_is_not_finite():
    ralm = _ralm()
    R, V, k = 3, 97, 24
    g = torch.Generator(DEV).manual_seed(8)
    logits = torch.randn((R, V), generator=g, device=DEV)
    ids, _, values = neighbours(R, V, k, 9)
    scores = 3.3e38 * (2.0 * torch.rand((R, k), generator=g, device=DEV) - 1.0)
    scores[:, 0], scores[:, 1] = 3.4e38, -3.4e38
    for metric, sign in ((ralm.IP, 1), (ralm.L2, -1)):
        for tau in (3e38, 1e38, 1e37):
            got = ralm.knn_mix(logits, ids, scores, values, 0.6, knn_temperature=tau, metric=metric)
            check(got, reference(logits, ids, scores, values, 0.6, 1.0, tau, sign))


def test_temperatures_whose_inverse_is_not_finite_are_refused():
    ralm = _ralm()
    logits, (ids, scores, values) = torch.randn((2, 50), device=DEV), neighbours(2, 50, 3, 7)
    for bad in (dict(temperature=1e-39), dict(knn_temperature=1e-39), dict(temperature=4e-39), dict(knn_temperature=1e-45)):
        with pytest.raises(ralm.RalmError) as e:
            ralm.knn_mix(logits, ids, scores, values, 0.5, **bad)
        assert e.value.status == 1
    check(ralm.knn_mix(logits, ids, scores, values, 0.5, temperature=5e-39, knn_temperature=5e-39),
          reference(logits, ids, scores, values, 0.5, 5e-39, 5e-39, -1))
