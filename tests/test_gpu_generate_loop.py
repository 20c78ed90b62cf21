"""The generator's operators together: the example's rounds of drafting, verifying and rolling back."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("knn_lm_speculation", os.path.join(ROOT, "examples", "knn_lm_speculation.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("branches", [False, True])
def test_rounds_of_speculation(branches):
    example = _example()
    out, history, cache = example.generate(requests=3, prompt=21, rounds=3, stride=3, branches=branches, seed=4)
    R = 6 if branches else 3
    assert len(history) == 3 and all(len(h) == R and all(0 <= a <= 3 for a in h) for h in history)
    assert [len(o) for o in out] == [21 + sum(1 + h[r] for h in history) for r in range(R)]
    # the rolled-back cache holds what a fresh pass over the same text puts there
    assert cache.lengths.tolist() == [len(o) for o in out]
    import paper_2401_14021_b200 as ralm
    fresh = ralm.KVCache.allocate(1, 2, 64, pages=64, rows=R, max_pages=8, page_size=16, device="cuda:0")
    fresh.resize(cache.lengths.clone())
    model = example.ToyModel(1000, heads=4, kv_heads=2, head_dim=64, seed=5, device="cuda:0")
    for r in range(R):
        row = torch.tensor([r], dtype=torch.int32, device="cuda:0")
        zero = torch.zeros(1, dtype=torch.int32, device="cuda:0")
        model.forward(fresh, torch.tensor([out[r]], device="cuda:0"), zero, rows=row)
        a, b = (c.read(0, zero, len(out[r]), rows=row) for c in (cache, fresh))
        # the projections of one token and of many may be rounded differently by the matrix library: one step of a code
        for x, y in zip(a, b):
            step = (y.float().amax(-1, keepdim=True) - y.float().amin(-1, keepdim=True)) / 15.0
            assert ((x.float() - y.float()).abs() <= 1.05 * step + 1e-2).all()
    # and the same seeds give the same tokens
    assert example.generate(requests=3, prompt=21, rounds=3, stride=3, branches=branches, seed=4)[0] == out


def test_target_alone_accepts_every_draft():
    """Without neighbours' share the drafts come from the target itself."""
    example = _example()
    _, history, _ = example.generate(requests=2, prompt=16, rounds=3, stride=4, lam=0.0, seed=5)
    # the two passes may round differently (a decode step and a pass over several tokens), so nearly all
    assert sum(map(sum, history)) >= 2 * 3 * 4 - 3
