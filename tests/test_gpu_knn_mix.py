"""The KNN-LM mixture against its definition in 64 bits.

Tolerance, set from the arithmetic: an exponent x log2(e) / T - r is rounded once at its own size (below 200
wherever the result is above 1e-60), 200 * 2^-24 * ln 2 = 8e-6 relative, and its factor log2(e) / T, the same for the whole
row, is within 2^-23 (below 2^22 powers of two; the rest is in test_gpu_knn_mix_extremes.py); the approximate 2^x adds
2^-22, the sums and the normalisation a few 2^-24. Neighbours: weights at 2^-22, their sum in 42-bit fixed point relative
to the token's largest. So 2e-5 relative."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
RTOL = 2e-5


def _ralm():
    import paper_2401_14021_b200 as ralm
    return ralm


def reference(logits, ids, scores, values, lam, T, tau, metric):
    R, V = logits.shape
    out = torch.zeros((R, V), dtype=torch.float64)
    for r in range(R):
        z = logits[r].double().cpu() / T
        lm = torch.zeros(V, dtype=torch.float64)
        some = bool((z > -math.inf).any() or z.isnan().any())
        if some:
            lm = torch.softmax(z, 0)
        knn, any_knn = torch.zeros(V, dtype=torch.float64), False
        if ids is not None:
            keep = [(values[i].item(), s) for i, s in zip(ids[r].tolist(), scores[r].double().tolist())
                    if 0 <= i < len(values) and math.isfinite(s) and 0 <= values[i].item() < V]
            if keep:
                any_knn = True
                w = torch.softmax(torch.tensor([(-s if metric else s) / tau for _, s in keep], dtype=torch.float64), 0)
                for (t, _), x in zip(keep, w):
                    knn[t] += x
        l = (lam if some else 1.0) if any_knn else 0.0
        out[r] = (1.0 - l) * lm + l * knn
    return out


def inputs(R, V, k, dtype, seed, N=1000, spread=3.0):
    g = torch.Generator(DEV).manual_seed(seed)
    logits = (spread * torch.randn((R, V), generator=g, device=DEV)).to(dtype)
    ids = torch.randint(-1, N, (R, k), generator=g, device=DEV)
    scores = 40.0 * torch.rand((R, k), generator=g, device=DEV)
    values = torch.randint(0, max(1, min(V, 50)), (N,), generator=g, device=DEV, dtype=torch.int32)   # many repeated tokens
    return logits, ids, scores, values


def check(got, want, rtol=RTOL):
    got = got.double().cpu()
    assert torch.equal(got.isnan(), want.isnan())
    ok = ~want.isnan()
    assert ((got - want).abs()[ok] <= rtol * want[ok] + 1e-37).all(), ((got - want).abs()[ok] / (want[ok] + 1e-37)).max()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,V,k", [(1, 1, 1), (2, 2, 0), (3, 7, 3), (1, 4097, 33), (5, 1000, 1024), (2, 32000, 8), (3, 50257, 1000),
                                   (700, 130, 5), (1, 131073, 20)])
def test_matches_definition(dtype, R, V, k):
    ralm = _ralm()
    logits, ids, scores, values = inputs(R, V, k, dtype, seed=V + k)
    for metric in (ralm.IP, ralm.L2):
        got = ralm.knn_mix(logits, ids, scores, values, 0.3, temperature=0.7, knn_temperature=8.0, metric=metric)
        check(got, reference(logits, ids, scores, values, 0.3, 0.7, 8.0, metric))


def test_row_too_long_for_shared_memory():
    ralm = _ralm()
    logits, ids, scores, values = inputs(2, 400_003, 9, torch.float32, seed=4)
    check(ralm.knn_mix(logits, ids, scores, values, 0.5), reference(logits, ids, scores, values, 0.5, 1.0, 1.0, 1))


@pytest.mark.parametrize("lam", [0.0, 1.0])
def test_lambda_at_its_ends(lam):
    ralm = _ralm()
    logits, ids, scores, values = inputs(4, 513, 20, torch.float16, seed=5)
    check(ralm.knn_mix(logits, ids, scores, values, lam), reference(logits, ids, scores, values, lam, 1.0, 1.0, 1))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_masked_and_odd_rows(dtype):
    ralm = _ralm()
    V = 3001
    logits, ids, scores, values = inputs(12, V, 12, dtype, seed=6)
    ids = ids.clamp(min=0)
    low = torch.finfo(dtype).min
    logits[0, :] = -math.inf                       # no token can come: the neighbours alone
    logits[1, :] = -math.inf
    ids[1, :] = -1                                 # ... and no neighbours: zeros
    ids[2, :] = -1                                 # no neighbours: the model alone
    logits[3, 1:] = -math.inf                      # one token left
    logits[4, :] = low                             # all at the type's lowest value: uniform
    logits[5, 5:] = low                            # masked by the lowest value
    logits[6, 7] = math.nan
    logits[7, 8] = math.inf
    scores[8, :6] = math.inf                       # padding of a short list
    scores[8, 6] = math.nan
    ids[9, 3] = 10 ** 12                           # outside the datastore
    values[ids[10, 0]] = -5                        # outside the vocabulary
    values[ids[10, 1]] = V
    logits[11, ::2] = -math.inf
    got = ralm.knn_mix(logits, ids, scores, values, 0.25, temperature=1.0, knn_temperature=5.0)
    want = reference(logits, ids, scores, values, 0.25, 1.0, 5.0, 1)
    assert (want[1] == 0).all() and want[6].isnan().all() and want[7].isnan().all()
    check(got, want)


def test_distances_that_agree_and_that_differ_widely():
    ralm = _ralm()
    logits, ids, scores, values = inputs(3, 257, 64, torch.float16, seed=7)
    scores[0, :] = 5.0
    scores[1, :] = torch.arange(64, device=DEV) * 1000.0
    scores[2, :] = -1e30
    check(ralm.knn_mix(logits, ids, scores, values, 0.9), reference(logits, ids, scores, values, 0.9, 1.0, 1.0, 1))


def test_row_pitches_and_alignment():
    ralm = _ralm()
    wide, ids, scores, values = inputs(9, 1203, 6, torch.float16, seed=8)
    out = torch.full((9, 1300), 7.0, device=DEV)
    for lo, hi, o in ((0, 1203, 0), (1, 1003, 3), (5, 1202, 1), (7, 8, 2)):
        got = ralm.knn_mix(wide[:, lo:hi], ids, scores, values, 0.3, probs=out[:, o:o + hi - lo])
        check(got, reference(wide[:, lo:hi], ids, scores, values, 0.3, 1.0, 1.0, 1))
        assert (out[:, :o] == 7.0).all() and (out[:, o + hi - lo:] == 7.0).all()     # nothing beside the rows is written
        out.fill_(7.0)


def test_one_bits_every_time_and_on_another_stream():
    ralm = _ralm()
    logits, ids, scores, values = inputs(40, 5000, 1024, torch.bfloat16, seed=9)
    values %= 3                                    # hundreds of neighbours per token
    first = ralm.knn_mix(logits, ids, scores, values, 0.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        again = ralm.knn_mix(logits, ids, scores, values, 0.5, stream=side)
        side.synchronize()
        assert torch.equal(first, again)


def test_without_neighbours_it_is_a_softmax():
    ralm = _ralm()
    logits = torch.randn((3, 999), device=DEV)
    got = ralm.knn_mix(logits, None, None, None, 0.5, temperature=2.0)
    check(got, torch.softmax(logits.double().cpu() / 2.0, 1))
    assert ralm.knn_mix(logits[:0], None, None, None, 0.5).shape == (0, 999)


def test_refusals():
    ralm = _ralm()
    logits, ids, scores, values = inputs(2, 100, 4, torch.float16, seed=10)
    for bad in (dict(lam=-0.1), dict(lam=1.1), dict(lam=math.nan), dict(temperature=0.0), dict(temperature=math.inf),
                dict(knn_temperature=-1.0), dict(metric=2)):
        with pytest.raises(ralm.RalmError) as e:
            ralm.knn_mix(logits, ids, scores, values, **{"lam": 0.5, **bad})
        assert e.value.status == 1
    for args in ((logits.int(), ids, scores, values), (logits, ids.int(), scores, values), (logits, ids, scores[:1], values),
                 (logits, ids, scores, values.long()), (logits.cpu(), ids, scores, values), (logits.t(), ids, scores, values)):
        with pytest.raises(TypeError):
            ralm.knn_mix(*args, 0.5)
    big = torch.zeros((1, 1025), dtype=torch.int64, device=DEV)
    with pytest.raises(ralm.RalmError):
        ralm.knn_mix(logits[:1], big, big.float(), values, 0.5)                     # more neighbours than a search returns
    with pytest.raises(TypeError):
        ralm.knn_mix(logits, ids, scores, values, 0.5, probs=torch.empty((2, 100), dtype=torch.float16, device=DEV))
    same = logits.float()
    with pytest.raises(ralm.RalmError):
        ralm.knn_mix(same, ids, scores, values, 0.5, probs=same)                   # in place
