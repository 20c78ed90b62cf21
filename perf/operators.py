"""What is measured of the generator-side operators: the KNN-LM mixture, the verification of drafted
tokens, the pages of a key-value cache, and the 4-bit cache with the attention that reads it.

Every case runs in two forms. The plain one computes the operator with elementary torch operations
in 32 bits; the other makes the calls of paper_2401_14021_b200 that a serving program makes. Both
take the same state, whose buffers are the program's own.

Layout of the 4-bit cache (one page holds `ps` tokens of every key-value head): per head
[K codes][V codes][K (scale, offset)][V (scale, offset)], ps * (D + 8) bytes. A token's vector x is
held as c = clamp(rint((x - b) / s) + 8, 0, 15) and stands for s * (c - 8) + b. K codes lie token by
token, two dimensions to a byte. V codes lie in blocks of 16 tokens: token 8c + 2t + e of the block
has dimension g + 8j as nibble j of the D / 16 bytes at [c][g][t][e].
"""
import math

import torch

own = False
DEV = "cuda"
LIMIT = 57344.0   # K and V values saturate here; NaN counts as zero


# ----------------------------------------------------------------------------- cases
def listed():
    return [
        # one request, OPT-sized vocabulary cut to LLaMA's, few neighbours: the latency of a decode step
        {"name": "mix_one_row", "op": "mix", "R": 1, "V": 32000, "k": 8, "dtype": "float16"},
        # 8 requests x stride 8 + 1, GPT-2's odd vocabulary, the KNN-LM evaluation's k = 1024
        {"name": "mix_verify_batch", "op": "mix", "R": 72, "V": 50257, "k": 1024, "dtype": "float16"},
        # 64 requests x stride 8, a large vocabulary
        {"name": "mix_large_vocab", "op": "mix", "R": 512, "V": 128000, "k": 64, "dtype": "bfloat16"},
        # one request with a stride of 4: the smallest verification
        {"name": "verify_one_request", "op": "verify", "R": 1, "S": 4, "V": 32000, "onehot": False},
        # 64 requests whose drafts come without probabilities, odd vocabulary
        {"name": "verify_onehot", "op": "verify", "R": 64, "S": 3, "V": 50257, "onehot": True},
        # 256 concurrent requests x stride 8
        {"name": "verify_batch", "op": "verify", "R": 256, "S": 8, "V": 128000, "onehot": False},
        # asynchronous verification of 16 requests: fork, grow both sides, roll back
        {"name": "pages_fork_grow", "op": "fork", "B": 16, "L": 24, "H": 8, "D": 64, "ps": 32, "M": 32, "n": 9},
        # a pool after many requests left: half the pages are live and move together
        {"name": "pages_compact", "op": "compact", "B": 64, "L": 32, "H": 8, "D": 128, "ps": 64, "P": 1024, "live": 512},
        # one token for each of 8 requests enters the cache
        {"name": "append_step", "op": "append", "B": 8, "n": 1, "H": 32, "D": 128, "ps": 32, "M": 40, "dtype": "float16"},
        # 16 retrieved documents of 509 tokens enter the cache
        {"name": "append_documents", "op": "append", "B": 16, "n": 509, "H": 32, "D": 128, "ps": 64, "M": 16, "dtype": "bfloat16"},
        # one request, one token, LLaMA-2-7B's heads, prompt and documents of 777 tokens
        {"name": "attend_one_token", "op": "attend", "B": 1, "n": 1, "H": 32, "G": 1, "D": 128, "ps": 32, "len": 777, "dtype": "float16"},
        # verification of 8 drafted tokens for 32 requests of ragged lengths, shared heads
        {"name": "attend_verify", "op": "attend", "B": 32, "n": 9, "H": 8, "G": 4, "D": 128, "ps": 64, "len": 32000, "dtype": "bfloat16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["mix", "verify", "fork", "compact", "append", "attend", "attend", "attend"])
    dtype = rng.choice(["float16", "bfloat16"])
    if op == "mix":
        V = _log(rng, 1000, 270000)
        return {"op": op, "R": max(1, min(_log(rng, 1, 512), 60_000_000 // V)), "V": V,
                "k": rng.choice([0, 1, 20, 256, 1000, 1024, _log(rng, 1, 1024)]), "dtype": rng.choice([dtype, "float32"])}
    if op == "verify":
        V, S = _log(rng, 1000, 200000), rng.randint(1, 16)
        return {"op": op, "R": max(1, min(_log(rng, 1, 256), 256_000_000 // (V * (S + 1)))), "S": S, "V": V, "onehot": rng.random() < 0.3}
    D, ps = rng.choice([64, 128]), rng.choice([16, 32, 64])
    if op == "fork":
        return {"op": op, "B": _log(rng, 1, 48), "L": rng.randint(1, 32), "H": rng.choice([1, 2, 5, 8]), "D": D, "ps": ps,
                "M": rng.randint(2, 40), "n": rng.randint(1, 17)}
    if op == "compact":
        P = _log(rng, 16, 1024)
        return {"op": op, "B": rng.randint(1, 64), "L": rng.randint(1, 32), "H": rng.choice([1, 2, 5, 8]), "D": D, "ps": ps,
                "P": P, "live": rng.randint(1, P - 1)}
    if op == "append":
        H, n = rng.choice([1, 5, 8, 12, 32]), _log(rng, 1, 700)
        B = max(1, min(_log(rng, 1, 64), 16 * 509 * 32 * 128 // (n * H * D)))
        return {"op": op, "B": B, "n": n, "H": H, "D": D, "ps": ps, "M": (n + rng.randint(0, 500)) // ps + 2, "dtype": dtype}
    H, G, n = rng.choice([1, 2, 5, 8, 16, 32]), rng.choice([1, 1, 3, 4, 8]), rng.choice([1, 1, 2, 5, 9])
    T = _log(rng, 1, 100000)
    B = max(1, min(_log(rng, 1, 96), 32 * 17000 * 8 * 128 // (T * H * D)))
    n = n if B * H * G * n * T <= 32 * 9 * 32 * 17000 else 1
    return {"op": op, "B": B, "n": n, "H": H, "G": G, "D": D, "ps": ps, "len": T, "dtype": dtype}


def work(case):
    op = case["op"]
    if op == "mix":
        e = 4 if case["dtype"] == "float32" else 2
        return {"bytes": case["R"] * (case["V"] * (e + 4) + 16 * case["k"]), "flops": 5 * case["R"] * case["V"]}
    if op == "verify":
        # one row of target and draft probabilities decides a request
        return {"bytes": case["R"] * case["V"] * (4 if case["onehot"] else 8), "flops": 4 * case["R"] * case["V"]}
    if op == "fork":
        # each of the B pairs copies the one page that both sides write to (if it is not full)
        return {"bytes": 2 * case["B"] * case["L"] * case["H"] * case["ps"] * (case["D"] + 8), "flops": 0}
    if op == "compact":
        # the live pages above the dense range: about live * (1 - live / P)
        moved = max(1, case["live"] * (case["P"] - case["live"]) // case["P"])
        return {"bytes": 2 * moved * case["L"] * case["H"] * case["ps"] * (case["D"] + 8), "flops": 0}
    if op == "append":
        # K and V in, 4-bit pages out, 4-bit pages in, K and V out
        vectors = 2 * case["B"] * case["n"] * case["H"]
        return {"bytes": vectors * (2 * 2 * case["D"] + 2 * (case["D"] // 2 + 4)), "flops": 8 * vectors * case["D"]}
    tokens = sum(_lengths(case))
    rows = case["n"] * case["G"]
    return {"bytes": tokens * case["H"] * (case["D"] + 8) + 4 * case["B"] * case["H"] * rows * case["D"],
            "flops": 4 * tokens * case["H"] * case["D"] * rows}


# ----------------------------------------------------------------------------- inputs
def _lengths(case):
    """Lengths of the requests in attention and append cases: from len / 16 to len, the longest first."""
    B, n, top = case["B"], case["n"], case.get("len", 0)
    return [max(min(n, top), int(top * (1.0 - 0.9375 * r / max(B - 1, 1)))) for r in range(B)]


def _gen(seed):
    return torch.Generator(DEV).manual_seed(int(seed))


def _rand(shape, g):
    return torch.rand(shape, generator=g, device=DEV)


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _page_bytes(case):
    return case["H"] * case["ps"] * (case["D"] + 8)


def prepare(case, seed):
    g = _gen(seed)
    state = {"case": case}
    op = case["op"]
    if op == "mix":
        R, V, k = case["R"], case["V"], case["k"]
        N = 1_000_000
        # a peaked distribution over the vocabulary and neighbours that mostly agree on a few tokens
        state["logits"] = (3.0 * _randn((R, V), g)).to(getattr(torch, case["dtype"]))
        zipf = (V ** _rand((N,), g)).long().clamp_(max=V) - 1
        state["values"] = zipf.to(torch.int32)
        ids = torch.randint(0, N, (R, k), generator=g, device=DEV)
        if k > 2:
            ids[:, 1::7] = -1                       # a search that found fewer than k rows
        state["ids"] = ids
        state["scores"] = (20.0 + 30.0 * _rand((R, k), g)).sort(1).values
        state["lam"], state["temperature"], state["tau"] = 0.25, 0.8, 10.0
        state["probs"] = torch.empty((R, V), device=DEV)
    elif op == "verify":
        R, S, V = case["R"], case["S"], case["V"]
        logits = 3.0 * _randn((R, S + 1, V), g)
        state["target"] = torch.softmax(logits, -1)
        draft = torch.softmax(logits[:, :S] + 0.5 * _randn((R, S, V), g), -1)
        state["tokens"] = torch.multinomial(draft.reshape(R * S, V), 1, generator=g).reshape(R, S)
        state["draft"] = None if case["onehot"] else draft
        state["uniforms"] = _rand((R, S + 1), g)
        state["draft_len"] = torch.randint(0, S + 1, (R,), generator=g, device=DEV, dtype=torch.int32)
        state["draft_len"][::2] = S
        state["out_tokens"] = torch.empty((R, S + 1), dtype=torch.int64, device=DEV)
        state["accepted"] = torch.empty((R,), dtype=torch.int32, device=DEV)
    elif op == "fork":
        B, M, ps, n = case["B"], case["M"], case["ps"], case["n"]
        top = max(1, M * ps - n)
        lengths = torch.randint(1, top + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        pages = (lengths + ps - 1) // ps
        P = B * M + 2 * B * ((n + ps - 1) // ps + 1)
        order = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
        table = torch.full((2 * B, M), -1, dtype=torch.int32, device=DEV)
        held = torch.arange(M, device=DEV)[None] < pages[:, None]
        table[:B] = torch.where(held, order[:B * M].reshape(B, M), -1)
        refs = torch.zeros(P, dtype=torch.int32, device=DEV)
        refs[table[:B][held].long()] = 1
        zero = torch.zeros_like(lengths)
        state.update(table=table, refs=refs, lengths=torch.cat([lengths, zero]),
                     src=torch.arange(B, device=DEV, dtype=torch.int32), dst=torch.arange(B, 2 * B, device=DEV, dtype=torch.int32),
                     grown=torch.cat([lengths + n, lengths + n]), back=torch.cat([lengths, zero]))
        state["pool"] = torch.randint(0, 256, (case["L"], P, _page_bytes(case)), generator=g, device=DEV, dtype=torch.uint8)
    elif op == "compact":
        B, P, live, ps = case["B"], case["P"], case["live"], case["ps"]
        M = -(-live // B)
        pages = torch.randperm(P, generator=g, device=DEV)[:live].to(torch.int32)
        table = torch.full((B * M,), -1, dtype=torch.int32, device=DEV)
        table[:live] = pages
        table = table.reshape(B, M)
        state["table0"], state["refs0"] = table, torch.zeros(P, dtype=torch.int32, device=DEV)
        state["refs0"][pages.long()] = 1
        state.update(table=table.clone(), refs=state["refs0"].clone(), lengths=((table >= 0).sum(1) * ps).to(torch.int32))
        state["pool"] = torch.randint(0, 256, (case["L"], P, _page_bytes(case)), generator=g, device=DEV, dtype=torch.uint8)
    elif op == "append":
        B, n, H, D, ps, M = (case[x] for x in ("B", "n", "H", "D", "ps", "M"))
        dtype = getattr(torch, case["dtype"])
        starts = torch.randint(0, M * ps - n + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        state.update(starts=starts, lengths=starts + n, refs=torch.ones(B * M, dtype=torch.int32, device=DEV),
                     table=torch.randperm(B * M, generator=g, device=DEV).to(torch.int32).reshape(B, M))
        state["pool"] = torch.zeros((1, B * M, _page_bytes(case)), dtype=torch.uint8, device=DEV)
        # keys have channels of their own size and offset, as trained heads do
        state["k"] = (_randn((B, n, H, D), g) * (0.3 + _rand((H, D), g)) + 0.5 * _randn((H, D), g)).to(dtype)
        state["v"] = _randn((B, n, H, D), g).to(dtype)
        state["k_back"], state["v_back"] = torch.empty_like(state["k"]), torch.empty_like(state["v"])
    else:
        B, n, H, D, ps, top = (case[x] for x in ("B", "n", "H", "D", "ps", "len"))
        M = -(-top // ps)
        lengths = _lengths(case)
        held = [-(-x // ps) for x in lengths]
        P = sum(held)
        order = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
        mask = torch.arange(M, device=DEV)[None] < _i32(held)[:, None]
        table = torch.full((B, M), -1, dtype=torch.int32, device=DEV)
        table[mask] = order
        pool = torch.empty((1, P, _page_bytes(case)), dtype=torch.uint8, device=DEV)
        scale, offset = 0.3 + _rand((H, 1, D), g), 0.5 * _randn((H, 1, D), g)
        for at in range(0, P, 4096):
            count = min(4096, P - at)
            kc = _quantise(_randn((count, H, ps, D), g) * scale + offset)
            vc = _quantise(_randn((count, H, ps, D), g))
            pool[0, at:at + count] = _pack(kc, vc)
        dtype = getattr(torch, case["dtype"])
        state.update(table=table, refs=torch.ones(P, dtype=torch.int32, device=DEV), lengths=_i32(lengths), pool=pool)
        state["q"] = (1.5 * _randn((B, n, H * case["G"], D), g)).to(dtype)
        state["out"] = torch.empty_like(state["q"])
    return state


# ----------------------------------------------------------------------------- the calls of the package
def _handle(state):
    """The cache handle over the program's tensors, made once as a serving program makes it."""
    if "handle" not in state:
        import paper_2401_14021_b200 as ralm
        case = state["case"]
        state["handle"] = ralm.KVCache(state["pool"], state["table"], state["lengths"], state["refs"],
                                       kv_heads=case["H"], head_dim=case["D"], page_size=case["ps"])
    return state["handle"]


def _run_own(state):
    import paper_2401_14021_b200 as ralm
    op = state["case"]["op"]
    if op == "mix":
        return {"probs": ralm.knn_mix(state["logits"], state["ids"], state["scores"], state["values"], state["lam"],
                                      temperature=state["temperature"], knn_temperature=state["tau"], probs=state["probs"])}
    if op == "verify":
        tokens, accepted = ralm.verify_tokens(state["tokens"], state["draft"], state["target"], state["uniforms"],
                                              draft_len=state["draft_len"], tokens=state["out_tokens"],
                                              accepted=state["accepted"])
        return {"tokens": tokens, "accepted": accepted}
    cache = _handle(state)
    if op == "fork":
        cache.fork(state["src"], state["dst"])
        cache.resize(state["grown"])
        grown = state["table"].clone()
        cache.resize(state["back"])
        return _pages_out(state, grown)
    if op == "compact":
        state["table"].copy_(state["table0"])
        state["refs"].copy_(state["refs0"])
        live = cache.compact()
        return {**_pages_out(state, None), "live": live}
    if op == "append":
        cache.append(0, state["k"], state["v"], state["starts"])
        k, v = cache.read(0, state["starts"], state["case"]["n"], k=state["k_back"], v=state["v_back"])
        return {"k": k, "v": v}
    return {"out": cache.attend(0, state["q"], out=state["out"])}


def _pages_out(state, grown):
    return {"table": state["table"], "lengths": state["lengths"], "refs": state["refs"], "pool": state["pool"], "grown": grown}


# ----------------------------------------------------------------------------- plain forms
def _quantise(x):
    """(codes, scale, offset) of vectors [..., D]: fp32 arithmetic, scale and offset held in 16 bits."""
    x = torch.nan_to_num(x.float(), nan=0.0).clamp(-LIMIT, LIMIT)
    lo, hi = x.amin(-1), x.amax(-1)
    s = ((hi - lo) * (1.0 / 15.0)).half()
    b = (lo + 8.0 * s.float()).half()
    inv = torch.where(s > 0, s.float().reciprocal(), 0.0)
    c = (torch.round((x - b.float()[..., None]) * inv[..., None]) + 8.0).clamp(0.0, 15.0)
    return c.to(torch.uint8), s, b


def _pairs(s, b):
    return torch.stack([s, b], -1).contiguous().view(torch.uint8).flatten(-2)


def _pack(kc, vc):
    """Page bytes [P][H * ps * (D + 8)] of whole pages: kc, vc are (codes, scale, offset) of [P][H][ps][D]."""
    (kq, ks, kb), (vq, vs, vb) = kc, vc
    P, H, ps, D = kq.shape
    k = (kq[..., 0::2] | kq[..., 1::2] << 4).reshape(P, H, -1)
    v = vq.reshape(P, H, ps // 16, 2, 4, 2, D // 8, 8).permute(0, 1, 2, 3, 7, 4, 5, 6)   # [c][g][t][e][j]
    v = (v[..., 0::2] | v[..., 1::2] << 4).reshape(P, H, -1)
    return torch.cat([k, v, _pairs(ks, kb).reshape(P, H, -1), _pairs(vs, vb).reshape(P, H, -1)], -1).reshape(P, -1)


def _fields(pages, H, ps, D):
    """Views of page bytes [..., H * ps * (D + 8)]: K codes, V codes, K pairs, V pairs."""
    x = pages.reshape(pages.shape[:-1] + (H, ps * (D + 8)))
    half = ps * D // 2
    pairs = x[..., 2 * half:].contiguous().view(torch.float16).reshape(x.shape[:-1] + (2, ps, 2)).float()
    return x[..., :half], x[..., half:2 * half], pairs[..., 0, :, :], pairs[..., 1, :, :]


def _nibbles(x):
    return torch.stack([x & 15, x >> 4], -1).flatten(-2).float() - 8.0


def _dequantise(pages, H, ps, D):
    """K and V values [..., H, ps, D] of page bytes."""
    kc, vc, kp, vp = _fields(pages, H, ps, D)
    lead = kc.shape[:-1]
    k = _nibbles(kc.reshape(lead + (ps, D // 2)))
    v = _nibbles(vc.reshape(lead + (ps // 16, 2, 8, 4, 2, D // 16)))       # [c][g][t][e][j]
    n = len(lead)
    v = v.permute(tuple(range(n)) + (n, n + 1, n + 3, n + 4, n + 5, n + 2)).reshape(lead + (ps, D))
    return k * kp[..., :1] + kp[..., 1:], v * vp[..., :1] + vp[..., 1:]


def _plain_mix(state):
    logits, ids, scores, values = state["logits"], state["ids"], state["scores"], state["values"]
    V = logits.shape[1]
    z = logits.float() / state["temperature"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(1, keepdim=True)
    lm = torch.where(total > 0, e / total, 0.0)
    if ids.shape[1] == 0:
        return {"probs": lm}
    token = values[ids.clamp(0, values.numel() - 1)].long()
    valid = (ids >= 0) & (ids < values.numel()) & (token >= 0) & (token < V) & torch.isfinite(scores)
    x = torch.where(valid, -scores / state["tau"], -math.inf)
    best = x.amax(1, keepdim=True)
    w = torch.exp(x - torch.where(best == -math.inf, 0.0, best))
    mass = w.sum(1, keepdim=True)
    lam = torch.where(mass > 0, torch.where(total > 0, state["lam"], 1.0), 0.0)
    w = torch.where(mass > 0, lam * w / mass, 0.0)
    return {"probs": ((1.0 - lam) * lm).scatter_add_(1, token.clamp(0, V - 1), w)}


def _weights(x):
    return (torch.nan_to_num(x, nan=0.0).clamp(0.0, 1.0) * float(1 << 40)).to(torch.int64)


def _plain_verify(state):
    tokens, draft, target, u = state["tokens"], state["draft"], state["target"], state["uniforms"]
    R, S = tokens.shape
    at = torch.arange(R, device=DEV)
    pos = torch.arange(S, device=DEV)[None]
    n = state["draft_len"].long().clamp(0, S)
    p = target[:, :S].gather(2, tokens[..., None])[..., 0]
    q = torch.ones_like(p) if draft is None else draft.gather(2, tokens[..., None])[..., 0]
    ok = (u[:, :S] * q < p) & (pos < n[:, None])
    accepted = ok.long().cumprod(1).sum(1)
    bonus = accepted >= n
    first = accepted.clamp(max=S - 1)
    prow = target[at, accepted]
    if draft is None:
        residual = prow.scatter(1, tokens[at, first][:, None], 0.0)
    else:
        residual = prow - draft[at, first]
    whole = _weights(prow)
    w = torch.where(bonus[:, None], whole, _weights(residual))
    w = torch.where(w.sum(1, keepdim=True) > 0, w, whole)
    total = w.sum(1)
    U = (u[:, S].double().clamp(0.0, 1.0) * 16777216.0).long().clamp(max=16777215)
    t = U * (total >> 32) * 256 + (U * (total & 0xFFFFFFFF) >> 24)
    token = (w.cumsum(1) <= t[:, None]).sum(1)
    token = torch.where(total > 0, token, -1)
    pos = torch.arange(S + 1, device=DEV)[None]
    out = torch.where(pos < accepted[:, None], torch.cat([tokens, tokens[:, :1]], 1), -1)
    out = torch.where(pos == accepted[:, None], token[:, None], out)
    return {"tokens": out, "accepted": accepted.int()}


def _plain_resize(state, new):
    table, lengths, refs, pool, ps = state["table"], state["lengths"], state["refs"], state["pool"], state["case"]["ps"]
    R, M = table.shape
    P = refs.numel()
    col = torch.arange(M, device=DEV)[None]
    row = torch.arange(R, device=DEV)
    have, need = (lengths + ps - 1) // ps, (new + ps - 1) // ps
    drop = (col >= need[:, None]) & (col < have[:, None])
    pages = table.clamp(min=0).long().flatten()
    refs.index_add_(0, pages, -drop.flatten().int())
    table.copy_(torch.where(drop, -1, table))
    # a page that the row goes on writing into, and that others hold too, is copied first
    last = table.gather(1, (lengths // ps).clamp(max=M - 1).long()[:, None])[:, 0].clamp(min=0).long()
    writes = (new > lengths) & (lengths % ps != 0)
    growers = torch.zeros(P, dtype=torch.int32, device=DEV).index_add_(0, last, writes.int())
    lowest = torch.full((P,), R, device=DEV).scatter_reduce_(0, last, torch.where(writes, row, R), "amin")
    keeps = (refs[last] == growers[last]) & (lowest[last] == row)
    cow = writes & (refs[last] > 1) & ~keeps
    more = (need - have).clamp(min=0)
    demand = more + cow.int()
    begin = demand.cumsum(0) - demand
    free = torch.argsort((refs != 0).int(), stable=True).int()
    fresh = free[begin.clamp(max=P - 1).long()]
    refs.index_add_(0, last, -cow.int())
    first = torch.where(new > lengths, have, M)[:, None]
    add = (col >= first) & (col < need[:, None])
    taken = free[(begin[:, None] + cow[:, None].int() + col - have[:, None]).clamp(0, P - 1).long()]
    table.copy_(torch.where(add, taken, table))
    table.copy_(torch.where(cow[:, None] & (col == (lengths // ps)[:, None]), fresh[:, None], table))
    refs.index_add_(0, free.long(), (torch.arange(P, device=DEV) < demand.sum()).int())
    pool[:, fresh[cow].long()] = pool[:, last[cow]]
    lengths.copy_(new)


def _plain_fork(state):
    table, lengths, refs, src, dst = state["table"], state["lengths"], state["refs"], state["src"].long(), state["dst"].long()
    refs.index_add_(0, table[dst].clamp(min=0).long().flatten(), -(table[dst] >= 0).int().flatten())
    refs.index_add_(0, table[src].clamp(min=0).long().flatten(), (table[src] >= 0).int().flatten())
    table[dst] = table[src]
    lengths[dst] = lengths[src]


def _plain_compact(state):
    table, refs, pool = state["table"], state["refs"], state["pool"]
    P = refs.numel()
    index = torch.arange(P, device=DEV)
    live = refs > 0
    n = live.sum()
    source, hole = (live & (index >= n)).nonzero()[:, 0], (~live & (index < n)).nonzero()[:, 0]
    place = index.clone()
    place[source] = hole
    pool[:, hole] = pool[:, source]
    refs[hole] = refs[source]
    refs[source] = 0
    table.copy_(torch.where(table >= 0, place[table.clamp(min=0).long()].int(), -1))
    return n.int().reshape(1)


def _plain_append(state):
    case, table, starts = state["case"], state["table"], state["starts"].long()
    n, H, D, ps = case["n"], case["H"], case["D"], case["ps"]
    dtype = state["k"].dtype
    where = starts[:, None] + torch.arange(n, device=DEV)[None]                       # [B][n]
    page = table.gather(1, where // ps).long()[..., None, None]
    slot = (where % ps)[..., None, None]
    head = torch.arange(H, device=DEV)[None, None, :, None]
    base = head * (ps * (D + 8))
    flat = state["pool"][0].reshape(-1)
    start = page * _page_bytes(case) + base
    byte = torch.arange(D // 2, device=DEV)
    (kq, ks, kb), (vq, vs, vb) = _quantise(state["k"]), _quantise(state["v"])
    flat[start + slot * (D // 2) + byte] = kq[..., 0::2] | kq[..., 1::2] << 4
    v = vq.reshape(vq.shape[:-1] + (D // 8, 8)).transpose(-1, -2)                     # [g][j]
    v = (v[..., 0::2] | v[..., 1::2] << 4).flatten(-2)
    s = slot % 16
    spot = (slot // 16) * (8 * D) + (s // 8) * (4 * D) + (byte // (D // 16)) * (D // 2) + (s % 8) // 2 * (D // 8) + s % 2 * (D // 16) + byte % (D // 16)
    flat[start + ps * (D // 2) + spot] = v
    four = torch.arange(4, device=DEV)
    flat[start + ps * D + 4 * slot + four] = _pairs(ks[..., None], kb[..., None])
    flat[start + ps * (D + 4) + 4 * slot + four] = _pairs(vs[..., None], vb[..., None])
    # and back again as values
    k = _nibbles(flat[start + slot * (D // 2) + byte])
    v = _nibbles(flat[start + ps * (D // 2) + spot])
    v = v.reshape(v.shape[:-1] + (8, D // 8)).transpose(-1, -2).flatten(-2)
    kp = flat[start + ps * D + 4 * slot + four].view(torch.float16).float()
    vp = flat[start + ps * (D + 4) + 4 * slot + four].view(torch.float16).float()
    return {"k": (k * kp[..., :1] + kp[..., 1:]).to(dtype), "v": (v * vp[..., :1] + vp[..., 1:]).to(dtype)}


def _plain_attend(state):
    case, q, table, lengths = state["case"], state["q"], state["table"], state["lengths"]
    B, n, H, G, D, ps = (case[x] for x in ("B", "n", "H", "G", "D", "ps"))
    k, v = _dequantise(state["pool"][0][table.clamp(min=0).long()], H, ps, D)         # [B][M][H][ps][D]
    k = k.transpose(1, 2).reshape(B, H, -1, D)
    v = v.transpose(1, 2).reshape(B, H, -1, D)
    x = q.float().reshape(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    scores = x @ k.transpose(2, 3) * (D ** -0.5)
    del k
    last = lengths[:, None] - n + torch.arange(n, device=DEV)[None]                    # [B][n]: the newest key that is seen
    seen = torch.arange(scores.shape[3], device=DEV)[None, None] <= last[..., None]    # [B][n][T]
    seen = seen.repeat_interleave(G, 1)[:, None]
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(3, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    del scores
    total = e.sum(3, keepdim=True)
    o = torch.where(total > 0, e @ v / total, 0.0)
    return {"out": o.reshape(B, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, H * G, D).to(q.dtype)}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "mix":
        return _plain_mix(state)
    if op == "verify":
        return _plain_verify(state)
    if op == "fork":
        _plain_fork(state)
        _plain_resize(state, state["grown"])
        grown = state["table"].clone()
        _plain_resize(state, state["back"])
        return _pages_out(state, grown)
    if op == "compact":
        state["table"].copy_(state["table0"])
        state["refs"].copy_(state["refs0"])
        live = _plain_compact(state)
        return {**_pages_out(state, None), "live": live}
    if op == "append":
        return _plain_append(state)
    return _plain_attend(state)


# ----------------------------------------------------------------------------- definitions in 64 bits
def exact(case, seed):
    op = case["op"]
    if op not in ("mix", "append", "attend"):
        return None                                # whole numbers
    state = prepare(case, seed)
    if op == "mix":
        rows = []
        for r in range(case["R"]):
            p = torch.softmax(state["logits"][r].double() / state["temperature"], 0)
            i = state["ids"][r]
            keep = i >= 0
            if keep.any():
                w = torch.softmax(-state["scores"][r][keep].double() / state["tau"], 0)
                p = (1 - state["lam"]) * p
                p.index_put_((state["values"][i[keep]].long(),), state["lam"] * w, accumulate=True)
            rows.append(p)
        return {"probs": torch.stack(rows)}
    if op == "append":
        return {name: _roundtrip(state[name].double()) for name in ("k", "v")}
    B, n, H, G, D, ps = (case[x] for x in ("B", "n", "H", "G", "D", "ps"))
    size = ps * (D + 8)
    d, t = torch.arange(D, device=DEV), torch.arange(ps, device=DEV)
    # where each code of a page's head lies: (byte, shift)
    kbyte = t[:, None] * (D // 2) + d[None] // 2
    kshift = (d[None] % 2 * 4).expand(ps, D)
    j, lane = d // 8, d % 8 * 4
    vbyte = ps * D // 2 + (t // 16 * 16 * D // 2 + t % 16 // 8 * 4 * D)[:, None] \
        + (lane[None] + (t % 8 // 2)[:, None]) * (D // 8) + (t % 2 * (D // 16))[:, None] + (j // 2)[None]
    vshift = (j % 2 * 4)[None].expand(ps, D)
    out = torch.zeros((B, n, H * G, D), dtype=torch.float64, device=DEV)
    for r, length in enumerate(_lengths(case)):
        pages = state["pool"][0][state["table"][r, :-(-length // ps)].long()].reshape(-1, H, size)
        for h in range(H):
            x = pages[:, h]
            pair = x[:, ps * D:].contiguous().view(torch.float16).double().reshape(-1, 2, ps, 2)
            k = ((x[:, kbyte] >> kshift & 15).double() - 8) * pair[:, 0, :, :1] + pair[:, 0, :, 1:]
            v = ((x[:, vbyte] >> vshift & 15).double() - 8) * pair[:, 1, :, :1] + pair[:, 1, :, 1:]
            k, v = k.reshape(-1, D)[:length], v.reshape(-1, D)[:length]
            for i in range(n):
                seen = length - n + i + 1
                if seen > 0:
                    z = state["q"][r, i, h * G:(h + 1) * G].double() @ k[:seen].T / math.sqrt(D)
                    out[r, i, h * G:(h + 1) * G] = torch.softmax(z, 1) @ v[:seen]
    return {"out": out}


def _roundtrip(x):
    """What a vector stands for once it is held in 4 bits, its scale and offset in 16."""
    low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
    s = ((high - low) / 15).half().double()
    b = (low + 8 * s).half().double()
    c = torch.where(s > 0, ((x - b) / s).round(), 0.0).clamp(-8, 7)
    return c * s + b
