"""Token-level speculation with a KNN-LM target, on the library's operators end to end.

A toy causal model (random weights: embedding, one attention layer over the 4-bit cache, tied output layer) stands
in for the generator. Each round, for every request at once:

  draft   `stride` tokens from the model alone, one decode step each: resize, append, attend, knn_mix (softmax)
  verify  one pass over the drafts (stride + 1 queries per request), the KNN-LM mixture with the neighbours that an
          exact search over the datastore returns, verify_tokens; then roll back: resize to the accepted length
  fork    (--branches) every request is forked for a second continuation, which shares its pages until they differ

    python examples/knn_lm_speculation.py --rounds 4
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2401_14021_b200 as ralm


class ToyModel:
    def __init__(self, vocab, heads, kv_heads, head_dim, seed, device):
        g = torch.Generator(device).manual_seed(seed)
        d = heads * head_dim
        rand = lambda *shape: torch.randn(shape, generator=g, device=device, dtype=torch.float32)  # noqa: E731
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.embed = rand(vocab, d).half()
        self.wq, self.wk, self.wv, self.wo = ((rand(d, n) * d ** -0.5).half() for n in
                                              (d, kv_heads * head_dim, kv_heads * head_dim, d))

    def forward(self, cache, tokens, starts, rows=None, q_len=None):
        """tokens [R][n] at positions starts[r] ..: their K and V enter the cache (whose rows are long enough),
        and logits [R][n][V] and hidden states [R][n][d] come back."""
        x = self.embed[tokens]
        shape = tokens.shape + (-1, self.head_dim)
        cache.append(0, (x @ self.wk).reshape(shape), (x @ self.wv).reshape(shape), starts, count=q_len, rows=rows)
        a = cache.attend(0, (x @ self.wq).reshape(shape), rows=rows, q_len=q_len)
        h = torch.nn.functional.normalize((x + a.reshape(x.shape) @ self.wo).float(), dim=-1).half()
        return 8.0 * (h @ torch.nn.functional.normalize(self.embed.float(), dim=-1).half().T), h


def generate(requests=4, prompt=33, rounds=4, stride=4, vocab=1000, entries=20000, k=32, lam=0.3, branches=False,
             seed=0, device="cuda:0"):
    """Returns (tokens of each request, accepted drafts of each round [rounds][requests], the cache)."""
    g = torch.Generator(device).manual_seed(seed)
    R = requests * (2 if branches else 1)
    most = prompt + rounds * (stride + 1) + stride + 1
    cache = ralm.KVCache.allocate(1, 2, 64, pages=R * (-(-most // 16) + 1), rows=R, max_pages=-(-most // 16) + 1,
                                  page_size=16, device=device)
    model = ToyModel(vocab, heads=4, kv_heads=2, head_dim=64, seed=seed + 1, device=device)
    # the datastore: hidden states of some text, and the token that followed each
    keys = torch.nn.functional.normalize(torch.randn((entries, 256), generator=g, device=device), dim=-1).half()
    values = torch.randint(0, vocab, (entries,), generator=g, device=device, dtype=torch.int32)
    index = ralm.Index(keys, ralm.L2, max_s=R * (stride + 1), max_k=k)

    lengths = torch.zeros(R, dtype=torch.int32, device=device)
    text = torch.randint(0, vocab, (requests, prompt), generator=g, device=device)
    lengths[:requests] = prompt
    cache.resize(lengths)
    rows = torch.arange(requests, dtype=torch.int32, device=device)
    zero = torch.zeros(requests, dtype=torch.int32, device=device)
    model.forward(cache, text, zero, rows=rows)
    if branches:
        cache.fork(rows, rows + requests)
        lengths[requests:] = prompt
        text = text.repeat(2, 1)
    out = [t.tolist() for t in text]
    newest = torch.randint(0, vocab, (R, 1), generator=g, device=device)   # each request's token that is not in the cache yet
    history = []
    for _ in range(rounds):
        # draft: decode steps of the model alone
        drafts, probs, token = [], [], newest
        for i in range(stride):
            cache.resize(lengths + (i + 1))
            logits, _ = model.forward(cache, token, lengths + i)
            p = ralm.knn_mix(logits[:, 0], None, None, None, 0.0)
            token = torch.multinomial(p, 1, generator=g)
            drafts.append(token)
            probs.append(p)
        cache.resize(lengths)                       # the drafts' K and V are computed again by the verification pass
        # verify: the newest token and the drafts in one pass, the mixture as the target
        step = torch.cat([newest] + drafts, 1)
        cache.resize(lengths + (stride + 1))
        logits, hidden = model.forward(cache, step, lengths)
        ids, dists = ralm.search(index, hidden.reshape(R * (stride + 1), -1).contiguous(), k)
        target = ralm.knn_mix(logits.reshape(-1, vocab), ids, dists, values, lam, knn_temperature=0.1)
        uniforms = torch.rand((R, stride + 1), generator=g, device=device)
        tokens, accepted = ralm.verify_tokens(torch.cat(drafts, 1), torch.stack(probs, 1),
                                              target.reshape(R, stride + 1, vocab), uniforms)
        # roll back to what stands: the newest token and the accepted drafts
        for r, t in enumerate(newest[:, 0].tolist()):
            out[r] += [t] + tokens[r, :accepted[r]].tolist()
        lengths = lengths + 1 + accepted
        cache.resize(lengths)
        newest = tokens.gather(1, accepted[:, None].long())
        history.append(accepted.tolist())
    if cache.device_status() != 0 or index.device_status() != 0:
        raise RuntimeError("a call was refused on the device")
    return out, history, cache


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--rounds", type=int, default=4)
    ap.add_argument("--stride", type=int, default=4)
    ap.add_argument("--branches", action="store_true")
    a = ap.parse_args()
    out, history, cache = generate(a.requests, rounds=a.rounds, stride=a.stride, branches=a.branches)
    for i, accepted in enumerate(history):
        print("round %d: accepted drafts %s" % (i, accepted))
    print("stride the scheduler would take next: %d" %
          ralm.os3_stride([x for h in history for x in h], [a.stride] * sum(map(len, history)), a=1.0, b=3.0))
    print("pages in use: %d, of them shared: %d" % ((cache.refs > 0).sum().item(), (cache.refs > 1).sum().item()))
