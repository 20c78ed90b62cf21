"""Results beside their inputs in one buffer; in place is refused (on the host)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def same_inputs_every_time():
    torch.manual_seed(0)


def test_columns_of_one_buffer():
    import paper_2401_14021_b200 as ralm
    both = torch.randn((7, 2006), generator=torch.Generator(DEV).manual_seed(1), device=DEV)
    logits, probs = both[:, :1003], both[:, 1003:]
    want = torch.softmax(logits.double(), 1)
    assert ralm.knn_mix(logits, None, None, None, 0.5, probs=probs) is probs
    assert ((probs.double() - want).abs() <= 2e-5 * want).all()      # the mixture's tolerance, see test_gpu_knn_mix.py
    with pytest.raises(ralm.RalmError):
        ralm.knn_mix(logits, None, None, None, 0.5, probs=both[:, 1002:2005])


def test_drafts_are_not_verified_in_place():
    import paper_2401_14021_b200 as ralm
    S, V = 4, 50
    tokens = torch.randint(0, V, (1, S + 1), device=DEV)
    target, u = torch.softmax(torch.randn((1, S + 1, V), device=DEV), -1), torch.rand((1, S + 1), device=DEV)
    lens = torch.tensor([3], dtype=torch.int32, device=DEV)
    before = tokens.clone()
    for kw in (dict(tokens=tokens), dict(accepted=lens)):
        with pytest.raises(ralm.RalmError) as e:
            ralm.verify_tokens(tokens[:, :S], None, target, u, draft_len=lens, **kw)
        assert e.value.status == 1
    assert torch.equal(tokens, before)
    ralm.verify_tokens(tokens[:, :S], None, target, u, draft_len=lens)


def test_attention_beside_its_queries():
    import paper_2401_14021_b200 as ralm
    cache = ralm.KVCache.allocate(1, 2, 64, pages=8, rows=2, max_pages=4, page_size=16, device=DEV)
    lengths = torch.tensor([20, 7], dtype=torch.int32, device=DEV)
    cache.resize(lengths)
    k = torch.randn((2, 20, 2, 64), device=DEV).half()
    cache.append(0, k, k, torch.zeros_like(lengths), count=lengths)
    both = torch.randn((2, 3, 8, 64), device=DEV).half()
    q, out = both[:, :, :4], both[:, :, 4:]
    want = cache.attend(0, q.clone())
    assert cache.attend(0, q, out=out) is out and torch.equal(out, want)
    for shifted in (both[:, :, 3:7], both[:, :, 1:5], q):
        with pytest.raises(ralm.RalmError):
            cache.attend(0, q, out=shifted)
    assert cache.device_status() == 0
