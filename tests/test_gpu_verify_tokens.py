"""Verification of drafted tokens, token for token, against the definition in Python's whole numbers."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ralm():
    import paper_2401_14021_b200 as ralm
    return ralm


def weights(x):
    """floor(2^40 min(max(x, 0), 1)), NaN as 0: exact in 64 bits, x has 24."""
    x = np.nan_to_num(np.asarray(x, np.float64), nan=0.0, posinf=1.0, neginf=0.0)
    return [int(v) for v in np.floor(np.clip(x, 0.0, 1.0) * 2.0 ** 40)]


def reference(tokens, draft, target, u, lens):
    R, S, V = tokens.shape[0], tokens.shape[1], target.shape[2]
    out, acc = [], []
    for r in range(R):
        n = S if lens is None else min(max(int(lens[r]), 0), S)
        a = 0
        while a < n:
            t = int(tokens[r, a])
            if not 0 <= t < V:
                break
            q = np.float32(1.0) if draft is None else draft[r, a, t]
            if not np.float32(u[r, a]) * q < target[r, a, t]:        # one product in 32 bits
                break
            a += 1
        row = target[r, a]
        with np.errstate(invalid="ignore"):
            if a < n and draft is not None:
                w = weights(row - draft[r, a])
            else:
                w = weights(row)
                if a < n and 0 <= int(tokens[r, a]) < V:
                    w[int(tokens[r, a])] = 0
        if sum(w) == 0:
            w = weights(row)
        T = sum(w)
        token = -1
        if T:
            us = float(u[r, S])
            us = 0.0 if math.isnan(us) else min(max(us, 0.0), 1.0)
            t = T * min(int(us * 2.0 ** 24), 2 ** 24 - 1) >> 24
            c = 0
            for v, x in enumerate(w):
                c += x
                if c > t:
                    token = v
                    break
        out.append([int(tokens[r, i]) for i in range(a)] + [token] + [-1] * (S - a))
        acc.append(a)
    return out, acc


def inputs(R, S, V, seed, closeness=0.5):
    g = torch.Generator(DEV).manual_seed(seed)
    logits = 3.0 * torch.randn((R, S + 1, V), generator=g, device=DEV)
    target = torch.softmax(logits, -1)
    draft = torch.softmax(logits[:, :S] + closeness * torch.randn((R, S, V), generator=g, device=DEV), -1)
    tokens = torch.multinomial(draft.reshape(R * S, V), 1, generator=g).reshape(R, S) if S else torch.empty((R, 0), dtype=torch.int64, device=DEV)
    u = torch.rand((R, S + 1), generator=g, device=DEV)
    return tokens, draft, target, u


def check(tokens, draft, target, u, lens=None):
    ralm = _ralm()
    got, acc = ralm.verify_tokens(tokens, draft, target, u, draft_len=lens)
    want, want_acc = reference(tokens.cpu().numpy(), None if draft is None else draft.cpu().numpy(), target.cpu().numpy(),
                               u.cpu().numpy(), None if lens is None else lens.cpu().numpy())
    assert acc.tolist() == want_acc
    assert got.tolist() == want
    return got, acc


@pytest.mark.parametrize("R,S,V", [(1, 1, 1), (1, 1, 2), (3, 4, 31), (2, 8, 257), (5, 3, 1000), (2, 4, 32000), (1, 16, 50257), (300, 2, 64),
                                   (2, 40, 100), (1, 2, 200_001)])
def test_matches_definition(R, S, V):
    tokens, draft, target, u = inputs(R, S, V, seed=R + S + V)
    check(tokens, draft, target, u)
    check(tokens, None, target, u)
    lens = torch.randint(-1, S + 2, (R,), device=DEV, dtype=torch.int32)
    check(tokens, draft, target, u, lens)
    check(tokens, None, target, u, lens)


def test_no_drafts():
    tokens, draft, target, u = inputs(4, 0, 500, seed=1)
    got, acc = check(tokens, None, target, u)
    assert got.shape == (4, 1) and acc.tolist() == [0] * 4


def test_identical_draft_and_target_accept_everything():
    tokens, _, target, u = inputs(6, 5, 300, seed=2)
    _, acc = check(tokens, target[:, :5].contiguous(), target, u)
    assert acc.tolist() == [5] * 6


def test_random_numbers_at_their_ends():
    tokens, draft, target, u = inputs(6, 4, 300, seed=3)
    u[0] = 0.0
    u[1] = 1.0 - 2.0 ** -24
    u[2] = 1.0                                     # outside [0, 1): held to it
    u[3] = -1.0
    u[4] = math.nan
    u[5, 4] = 2.0 ** -25
    check(tokens, draft, target, u)


def test_rows_with_nothing_left():
    tokens, draft, target, u = inputs(6, 2, 200, seed=4)
    u[:, :2] = 1.0
    draft[0] = target[0, :2] * 4.0                 # the draft covers the target everywhere: draw from the target
    target[1] = 0.0                                # no token has any probability
    target[2] = 0.0
    target[2, :, 199] = 1e-30                      # below a step of the fixed point
    target[3] = math.nan
    draft[4] = math.nan
    target[5] = math.inf                           # held to 1
    got, _ = check(tokens, draft, target, u)
    assert got[1].tolist() == [-1, -1, -1] and got[3, 0] == -1


def test_tokens_outside_the_vocabulary_are_rejected():
    tokens, draft, target, u = inputs(4, 3, 50, seed=5)
    tokens[0, 0], tokens[1, 1], tokens[2, 2] = -1, 50, 2 ** 40
    check(tokens, draft, target, u)
    check(tokens, None, target, u)


def test_every_token_is_drawn_in_its_share():
    """All 2^12 evenly spaced random numbers through one row: each token comes floor or ceil of its share."""
    ralm = _ralm()
    V, n = 37, 4096
    g = torch.Generator(DEV).manual_seed(6)
    row = torch.softmax(2.0 * torch.randn(V, generator=g, device=DEV), 0)
    target = row.expand(n, 1, V)                   # one row for all, by a stride of zero
    u = (torch.arange(n, device=DEV, dtype=torch.float32) / n).reshape(n, 1)
    got, _ = ralm.verify_tokens(torch.empty((n, 0), dtype=torch.int64, device=DEV), None, target, u)
    counts = torch.bincount(got[:, 0], minlength=V).double().cpu()
    share = row.double().cpu() / row.double().sum().cpu() * n
    assert (counts.sum() == n) and ((counts - share).abs() < 1.0 + 1e-6).all()


def test_strides_and_alignment():
    ralm = _ralm()
    R, S, V = 5, 3, 203
    tokens, draft, target, u = inputs(R, S, V, seed=7)
    wide_t = torch.zeros((R, S + 3, V + 9), device=DEV)
    wide_d = torch.zeros((S, R, V + 2), device=DEV)
    wide_t[:, 1:S + 2, 5:5 + V] = target
    wide_d[:, :, 1:1 + V] = draft.transpose(0, 1)
    a = ralm.verify_tokens(tokens, draft, target, u)
    b = ralm.verify_tokens(tokens, wide_d[:, :, 1:1 + V].transpose(0, 1), wide_t[:, 1:S + 2, 5:5 + V], u)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_largest_sums_do_not_overflow():
    """Rows that are no distribution: every weight at its largest, more terms than one 32-bit sum holds."""
    V = 4200 * 512
    target = torch.ones((1, 1, V), device=DEV)
    for x in (0.0, 0.25, 0.999999):
        u = torch.tensor([[x]], device=DEV)
        got, _ = _ralm().verify_tokens(torch.empty((1, 0), dtype=torch.int64, device=DEV), None, target, u)
        assert got.item() == V * int(x * 2 ** 24 + 0.0) // 2 ** 24 if x != 0.999999 else abs(got.item() - x * V) < 2


def test_feeds_the_stride_scheduler():
    ralm = _ralm()
    tokens, draft, target, u = inputs(8, 4, 500, seed=8)
    _, acc = ralm.verify_tokens(tokens, draft, target, u)
    gamma = ralm.os3_gamma(acc.tolist(), [4] * 8)
    assert 0.0 <= gamma <= 0.6


def test_refusals():
    ralm = _ralm()
    tokens, draft, target, u = inputs(2, 3, 40, seed=9)
    for args in ((tokens.int(), draft, target, u), (tokens, draft[:, :2], target, u), (tokens, draft.half(), target, u),
                 (tokens, draft, target[:, :3], u), (tokens, draft, target, u[:, :3]), (tokens, draft, target, u.double()),
                 (tokens.cpu(), draft, target, u), (tokens, draft, target.transpose(1, 2), u)):
        with pytest.raises(TypeError):
            ralm.verify_tokens(*args)
    with pytest.raises(TypeError):
        ralm.verify_tokens(tokens, draft, target, u, draft_len=torch.zeros(2, dtype=torch.int64, device=DEV))
    with pytest.raises(ralm.RalmError):
        ralm.verify_tokens(tokens[:, :0].contiguous(), None, target[:, :1, :0], u[:, :1].contiguous())   # an empty vocabulary
    empty = ralm.verify_tokens(tokens[:0], None, target[:0], u[:0])
    assert empty[0].shape == (0, 4)
