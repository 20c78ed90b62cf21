"""The 4-bit cache: append and read against the format's definition, attention against 64 bits.

Attention's tolerance, set from the arithmetic: with k and v the values that the codes stand for, scores are exact up
to a few 2^-24 of sum |q k| (below 1e-4 here); the weights are rounded to fp16 (2^-12 of each at most, taken as 2^-11),
the result to its type (2^-11 fp16, 2^-8 bf16). So each output is within (2^-11 + u + 1e-4) sum p (|v| + |b|) of the
definition, b being the offset of v, which enters the sum by itself."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LIMIT = np.float32(57344.0)


def _ralm():
    import paper_2401_14021_b200 as ralm
    return ralm


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def stands_for(x):
    """What vectors [..., D] stand for once they are held: (values in 64 bits, s, b), from the format's definition."""
    x = x.float().cpu().numpy()
    x = np.clip(np.where(np.isnan(x), np.float32(0), x), -LIMIT, LIMIT)
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    s = ((hi - lo) * np.float32(1.0 / 15.0)).astype(np.float16).astype(np.float32)
    b = (lo + np.float32(8) * s).astype(np.float16).astype(np.float32)
    with np.errstate(divide="ignore"):
        inv = np.where(s > 0, np.float32(1) / s, np.float32(0)).astype(np.float32)
    c = np.clip(np.rint((x - b) * inv), -8, 7)
    return c.astype(np.float64) * s + b, s.astype(np.float64), b.astype(np.float64)


def make_cache(B, heads, D, ps, max_pages, layers=1, spare=3, seed=0, poison=True):
    ralm = _ralm()
    cache = ralm.KVCache.allocate(layers, heads, D, B * max_pages + spare, B, max_pages, ps, device=DEV)
    if poison:
        cache.pool.fill_(0xFF)                     # every scale and offset that was not written is a NaN
    # pages in no order
    g = torch.Generator(DEV).manual_seed(seed)
    order = torch.randperm(B * max_pages + spare, generator=g, device=DEV).to(torch.int32)
    return cache, order


def give_pages(cache, order, lengths):
    ps, at = cache.page_size, 0
    cache.table.fill_(-1)
    cache.refs.zero_()
    for r, n in enumerate(lengths):
        need = -(-n // ps)
        cache.table[r, :need] = order[at:at + need]
        at += need
    cache.refs[order[:at].long()] = 1
    cache.lengths.copy_(i32(lengths))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ps,B,H,n", [(16, 1, 1, 1), (16, 3, 5, 17), (32, 2, 2, 100), (64, 4, 3, 70), (64, 2, 32, 9)])
def test_append_and_read(dtype, D, ps, B, H, n):
    g = torch.Generator(DEV).manual_seed(n)
    cache, order = make_cache(B, H, D, ps, max_pages=(n + 90) // ps + 2, layers=2, seed=n)
    starts = [(7 * r + 3) % 81 for r in range(B)]
    give_pages(cache, order, [s + n for s in starts])
    k = (torch.randn((B, n, H, D), generator=g, device=DEV) * (0.2 + torch.rand((H, D), generator=g, device=DEV)) + 3.0).to(dtype)
    v = torch.randn((B, n, H, D), generator=g, device=DEV).to(dtype)
    before = cache.pool[0].clone()
    cache.append(1, k, v, i32(starts))
    assert torch.equal(cache.pool[0], before)      # the other layer
    bk, bv = cache.read(1, i32(starts), n, dtype=dtype)
    assert cache.device_status() == 0
    for x, back in ((k, bk), (v, bv)):
        want, s, _ = stands_for(x)
        got = back.double().cpu().numpy()
        u = 2.0 ** -11 if dtype is torch.float16 else 2.0 ** -8
        assert (np.abs(got - want) <= u * np.abs(want) + 1e-7).all()           # the format, rounded once
        xs = x.double().cpu().numpy()
        # and near what came in: half a step, plus what the offset's 11 bits moved the range by, plus the rounding
        assert (np.abs(got - xs) <= 0.5 * s + 2.0 ** -11 * (np.abs(xs).max(-1, keepdims=True) + 8 * s) + u * np.abs(want) + 1e-6).all()


@pytest.mark.parametrize("D", [64, 128])
def test_append_touches_only_its_tokens(D):
    H, ps = 2, 16
    cache, order = make_cache(2, H, D, ps, 6, seed=3)
    give_pages(cache, order, [60, 40])
    g = torch.Generator(DEV).manual_seed(1)
    k = torch.randn((2, 60, H, D), generator=g, device=DEV).half()
    v = torch.randn((2, 60, H, D), generator=g, device=DEV).half()
    cache.append(0, k, v, i32([0, 0]), count=i32([60, 40]))
    k0, v0 = cache.read(0, i32([0, 0]), 60)
    assert (k0[1, 40:] == 0).all() and (v0[1, 40:] == 0).all()                    # beyond the row's length
    for start, n in ((0, 1), (15, 1), (16, 1), (31, 2), (14, 5), (33, 20)):
        x = torch.randn((1, n, H, D), generator=g, device=DEV).half()
        y = torch.randn((1, n, H, D), generator=g, device=DEV).half()
        cache.append(0, x, y, i32([start]), rows=i32([0]))
        k1, v1 = cache.read(0, i32([0, 0]), 60)
        kw, vw = cache.read(0, i32([start]), n, rows=i32([0]))
        k0[0, start:start + n], v0[0, start:start + n] = kw[0], vw[0]
        assert torch.equal(k1, k0) and torch.equal(v1, v0)
        assert (np.abs(kw[0].double().cpu().numpy() - stands_for(x[0])[0]) <= 2.0 ** -11 * 8).all()
    assert cache.device_status() == 0


def test_vectors_that_are_odd():
    D, H = 64, 9
    cache, order = make_cache(1, H, D, 16, 1)
    give_pages(cache, order, [16])
    x = torch.randn((1, 1, H, D), device=DEV).bfloat16()
    x[0, 0, 0] = 0.0                                # a scale of zero
    x[0, 0, 1] = -3.5                               # constant
    x[0, 0, 2, 5] = float("nan")                    # counts as 0
    x[0, 0, 3, 5] = float("inf")                    # saturates
    x[0, 0, 4, 5] = -1e30
    x[0, 0, 5] = float("nan")
    x[0, 0, 6] *= 1e-30                             # below what 16 bits hold
    x[0, 0, 7] = 1000.0 + x[0, 0, 7] * 0.01         # the offset's rounding moves the range
    x[0, 0, 8, 0], x[0, 0, 8, 1] = 57344.0, -57344.0
    cache.append(0, x, x, i32([4]))
    k, v = cache.read(0, i32([4]), 1, dtype=torch.bfloat16)
    want = stands_for(x)[0]
    for got in (k, v):
        got = got.double().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1e-7).all()
    assert cache.device_status() == 0


def test_strided_inputs():
    B, n, H, D = 2, 19, 3, 128
    cache, order = make_cache(B, H, D, 32, 2)
    give_pages(cache, order, [n, n])
    fused = torch.randn((B, n, 3 * H * D + 1), device=DEV).half()
    k = fused[:, :, H * D:2 * H * D].unflatten(2, (H, D))
    v = fused[:, :, 2 * H * D + 1:].unflatten(2, (H, D))         # rows that are not 16-byte aligned
    cache.append(0, k, v, i32([0, 0]))
    a = cache.read(0, i32([0, 0]), n)
    cache.pool.zero_()
    cache.append(0, k.contiguous(), v.contiguous(), i32([0, 0]))
    b = cache.read(0, i32([0, 0]), n)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    wide = torch.full((B, n, H, D + 1), 9.0, device=DEV).half()
    cache.read(0, i32([0, 0]), n, k=wide[..., 1:], v=torch.empty_like(v))
    assert torch.equal(wide[..., 1:], b[0]) and (wide[..., 0] == 9.0).all()


def test_append_leaves_out_what_it_may_not_write():
    H, D, ps = 1, 64, 16
    cache, order = make_cache(3, H, D, ps, 4)
    give_pages(cache, order, [20, 20, 0])
    x = torch.randn((3, 4, H, D), device=DEV).half()
    cache.append(0, x[:1], x[:1], i32([18]), rows=i32([0]))      # two of the four lie beyond the row
    assert cache.device_status() == 1
    assert (cache.read(0, i32([18]), 4, rows=i32([0]))[0][0, 2:] == 0).all()
    before = cache.pool.clone()
    for rows, starts in (([3], [0]), ([-1], [0]), ([0], [20]), ([2], [0]), ([0], [-4])):
        cache.append(0, x[:1], x[:1], i32(starts), rows=i32(rows))
        assert cache.device_status() == 1
    cache.fork(i32([0]), i32([2]))                               # now shared: read, but not written
    cache.append(0, x[:1], x[:1], i32([16]), rows=i32([2]))
    assert cache.device_status() == 1 and torch.equal(cache.pool, before)
    cache.resize(i32([20, 20, 24]))                              # copy on write
    cache.append(0, x[:1], x[:1], i32([20]), rows=i32([2]))
    assert cache.device_status() == 0
    a, b = cache.read(0, i32([18]), 2, rows=i32([0])), cache.read(0, i32([18]), 2, rows=i32([2]))   # the two that were written
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    cache.table[0, 0] = 10 ** 6                                   # a page number outside the pool
    cache.append(0, x[:1], x[:1], i32([0]), rows=i32([0]))
    assert cache.device_status() == 1
    cache.read(0, i32([0]), 4, rows=i32([0]))
    assert cache.device_status() == 1


# --------------------------------------------------------------------------------- attention
def filled(B, H, D, ps, lengths, seed, layers=1, max_pages=None):
    """A cache whose rows hold random tokens, and (k, v, offsets of v) as they stand, in 64 bits, [B][T][H][D]."""
    top = max(max(lengths), 1)
    cache, order = make_cache(B, H, D, ps, max_pages or -(-top // ps), layers=layers, seed=seed)
    give_pages(cache, order, lengths)
    g = torch.Generator(DEV).manual_seed(seed)
    k = (torch.randn((B, top, H, D), generator=g, device=DEV) * (0.3 + torch.rand((H, D), generator=g, device=DEV))
         + 0.5 * torch.randn((H, D), generator=g, device=DEV)).half()
    v = (torch.randn((B, top, H, D), generator=g, device=DEV) * torch.rand((B, top, H, 1), generator=g, device=DEV) + 0.2).half()
    cache.append(layers - 1, k, v, i32([0] * B), count=i32(lengths))
    assert cache.device_status() == 0
    dk, _, _ = stands_for(k)
    dv, _, bv = stands_for(v)
    return cache, torch.from_numpy(dk).to(DEV), torch.from_numpy(dv).to(DEV), torch.from_numpy(bv).to(DEV)


def attend_reference(q, k, v, b, lengths, scale, q_len=None):
    """(out, sum p (|v| + |b|)) in 64 bits."""
    B, n, Hq, D = q.shape
    G = Hq // k.shape[2]
    out = torch.zeros((B, n, Hq, D), dtype=torch.float64, device=DEV)
    size = torch.zeros_like(out)
    for r in range(B):
        m = n if q_len is None else min(max(q_len[r], 0), n)
        for i in range(m):
            seen = lengths[r] - m + i + 1
            if seen <= 0:
                continue
            for h in range(k.shape[2]):
                z = q[r, i, h * G:(h + 1) * G].double() @ k[r, :seen, h].T * scale
                p = torch.softmax(z, 1)
                out[r, i, h * G:(h + 1) * G] = p @ v[r, :seen, h]
                size[r, i, h * G:(h + 1) * G] = p @ (v[r, :seen, h].abs() + b[r, :seen, h].abs())
    return out, size


def check(got, want, size):
    u = 2.0 ** -11 if got.dtype is torch.float16 else 2.0 ** -8
    assert not got.isnan().any()
    off = (got.double() - want).abs()
    bound = (2.0 ** -11 + u + 1e-4) * size + 1e-7
    assert (off <= bound).all(), (off / bound).max()
    assert (got[size.sum(-1) == 0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ps", [16, 32, 64])
@pytest.mark.parametrize("n,H,G,lengths", [(1, 1, 1, [1]), (1, 2, 1, [0, 1, 15, 16, 17, 63, 64, 65, 200]), (3, 2, 4, [0, 1, 2, 3, 4, 130]),
                                           (9, 1, 2, [5, 9, 10, 1000]), (2, 3, 5, [33, 700]), (1, 1, 8, [5000]), (9, 2, 4, [300, 40]),
                                           (8, 1, 8, [77, 257])])
def test_attention_matches_definition(dtype, D, ps, n, H, G, lengths):
    cache, k, v, b = filled(len(lengths), H, D, ps, lengths, seed=n + H + G, layers=2)
    q = (1.5 * torch.randn((len(lengths), n, H * G, D), device=DEV)).to(dtype)
    got = cache.attend(1, q)
    assert cache.device_status() == 0
    check(got, *attend_reference(q, k, v, b, lengths, D ** -0.5))


def test_many_entries_of_any_length():
    """More entries than a CTA has threads, from nothing to some hundreds of tokens, all segments split differently."""
    g = np.random.RandomState(1)
    lengths = [int(x) for x in g.randint(0, 90, 900)]
    lengths[7], lengths[800] = 3000, 0
    cache, k, v, b = filled(900, 1, 64, 16, lengths, seed=5)
    for n, heads in ((1, 1), (2, 5)):
        q = torch.randn((900, n, heads, 64), device=DEV).half()
        got = cache.attend(0, q)
        assert cache.device_status() == 0
        check(got, *attend_reference(q, k, v, b, lengths, 0.125))


@pytest.mark.parametrize("n,G", [(1, 1), (5, 8)])
def test_one_long_row(n, G):
    cache, k, v, b = filled(1, 1, 128, 64, [70_001], seed=6)
    q = (2.0 * torch.randn((1, n, G, 128), device=DEV)).half()
    first = cache.attend(0, q)
    check(first, *attend_reference(q, k, v, b, [70_001], 128 ** -0.5))
    for _ in range(5):                             # whoever merges the pieces, the bits are the same
        assert torch.equal(cache.attend(0, q), first)


def test_ragged_queries_rows_and_scale():
    lengths = [40, 3, 100, 7]
    cache, k, v, b = filled(4, 2, 64, 32, lengths, seed=7)
    rows, q_len = [2, 0, 1, 2, 3], [0, 4, 5, 2, 9]
    q = torch.randn((5, 5, 6, 64), device=DEV).bfloat16()
    got = cache.attend(0, q, scale=0.3, rows=i32(rows), q_len=i32(q_len))
    assert cache.device_status() == 0
    check(got, *attend_reference(q, k[rows], v[rows], b[rows], [lengths[r] for r in rows], 0.3, q_len))
    got = cache.attend(0, q, scale=-0.3, rows=i32(rows))
    check(got, *attend_reference(q, k[rows], v[rows], b[rows], [lengths[r] for r in rows], -0.3))
    # rows outside the table: zeros, and the status word says so
    got = cache.attend(0, q, rows=i32([4, -1, 0, 1, 2]))
    assert cache.device_status() == 1 and (got[:2] == 0).all() and not (got[2] == 0).all()


def test_strided_queries_and_outputs():
    lengths = [50, 20]
    cache, k, v, b = filled(2, 2, 64, 16, lengths, seed=8)
    fused = torch.randn((2, 3, 8 * 64 + 1), device=DEV).half()
    for q in (fused[:, :, :256].unflatten(2, (4, 64)), fused[:, :, 1:257].unflatten(2, (4, 64)), fused[:, :, :256].unflatten(2, (4, 64)).transpose(1, 2).contiguous().transpose(1, 2)):
        wide = torch.full((2, 4, 3, 66), 5.0, device=DEV).half()
        out = wide[..., 1:65].transpose(1, 2)
        got = cache.attend(0, q, out=out)
        check(got, *attend_reference(q, k, v, b, lengths, 0.125))
        assert (wide[..., 0] == 5.0).all() and (wide[..., 65] == 5.0).all()


def test_queries_of_any_size():
    """Rows of one entry that differ by many powers of two, zero rows, and values beyond fp16 in bf16."""
    lengths = [90]
    cache, k, v, b = filled(1, 1, 128, 64, lengths, seed=9)
    q = torch.randn((1, 1, 8, 128), device=DEV)
    q *= torch.tensor([1.0, 0.0, 1e-3, 10.0, 1e-6, 30.0, 1e-2, 3.0], device=DEV)[:, None]
    check(cache.attend(0, q.half()), *attend_reference(q.half(), k, v, b, lengths, 128 ** -0.5))
    qb = (q * 1e5).bfloat16()
    check(cache.attend(0, qb, scale=1e-6), *attend_reference(qb, k, v, b, lengths, 1e-6))
    bad = q.half()
    bad[0, 0, 2, 5] = float("nan")
    bad[0, 0, 3, 5] = float("inf")
    got = cache.attend(0, bad)
    assert got[0, 0, 2].isnan().all() and got[0, 0, 3].isnan().all()
    rest = [0, 1, 4, 5, 6, 7]                      # the other rows are as they were
    want, size = attend_reference(q.half(), k, v, b, lengths, 128 ** -0.5)
    check(got[:, :, rest], want[:, :, rest], size[:, :, rest])


def test_values_whose_scales_differ_widely():
    """A token whose values are 10^4 times the others', early, late, and with little weight."""
    for at in (0, 40, 299):
        cache, order = make_cache(1, 1, 64, 32, 10)
        give_pages(cache, order, [300])
        k, v = torch.randn((1, 300, 1, 64), device=DEV).half(), torch.randn((1, 300, 1, 64), device=DEV).half()
        v[0, at] *= 1e4
        v[0, (at + 7) % 300] = 0.0
        v[0, (at + 9) % 300] = 2.5                 # a scale of zero
        cache.append(0, k, v, i32([0]))
        dk, dv, bv = (torch.from_numpy(x).to(DEV) for x in (stands_for(k)[0], stands_for(v)[0], stands_for(v)[2]))
        q = torch.randn((1, 1, 4, 64), device=DEV).half()
        check(cache.attend(0, q), *attend_reference(q, dk, dv, bv, [300], 0.125))


def test_scores_that_rise_and_fall():
    """Maxima that move by far more than the slack along the row, both ways."""
    lengths = [1500]
    for sign in (1.0, -1.0):
        cache, order = make_cache(1, 1, 64, 16, 94)
        give_pages(cache, order, lengths)
        ramp = torch.linspace(-20.0, 20.0, 1500, device=DEV)[None, :, None, None] * sign
        k = (torch.randn((1, 1500, 1, 64), device=DEV) * 0.1 + ramp).half()
        v = torch.randn((1, 1500, 1, 64), device=DEV).half()
        cache.append(0, k, v, i32([0]))
        dk, dv, bv = (torch.from_numpy(x).to(DEV) for x in (stands_for(k)[0], stands_for(v)[0], stands_for(v)[2]))
        q = (torch.rand((1, 3, 2, 64), device=DEV) + 0.5).half()
        check(cache.attend(0, q), *attend_reference(q, dk, dv, bv, lengths, 0.125))


def test_a_bad_page_number_is_reported():
    cache, k, v, b = filled(2, 1, 64, 16, [40, 40], seed=10)
    q = torch.randn((2, 1, 1, 64), device=DEV).half()
    good = cache.attend(0, q)
    cache.table[0, 1] = 10 ** 8
    got = cache.attend(0, q)
    assert cache.device_status() == 1 and torch.equal(got[1], good[1])


def test_offsets_beyond_32_bits():
    ralm = _ralm()
    H, D, ps = 8, 128, 64
    pages = 2 ** 32 // ralm.KVCache.page_bytes(H, D, ps) + 40
    cache = ralm.KVCache.allocate(1, H, D, pages, 1, 4, ps, device=DEV)          # 4.3 GB
    cache.table[0, :2] = i32([pages - 1, pages - 7])
    cache.refs[[pages - 1, pages - 7]] = 1
    cache.lengths.fill_(100)
    k, v = torch.randn((1, 100, H, D), device=DEV).half(), torch.randn((1, 100, H, D), device=DEV).half()
    cache.append(0, k, v, i32([0]))
    dk, dv, bv = (torch.from_numpy(x).to(DEV) for x in (stands_for(k)[0], stands_for(v)[0], stands_for(v)[2]))
    q = torch.randn((1, 2, 2 * H, D), device=DEV).half()
    check(cache.attend(0, q), *attend_reference(q, dk, dv, bv, [100], D ** -0.5))
    assert cache.device_status() == 0


def test_forked_rows_read_the_same_and_graphs_replay():
    cache, k, v, b = filled(2, 2, 64, 16, [50, 0], seed=11, max_pages=6)
    cache.refs.zero_()
    cache.refs[cache.table[cache.table >= 0].long()] = 1
    cache.fork(i32([0]), i32([1]))
    q = torch.randn((1, 1, 4, 64), device=DEV).half()
    q2 = q.expand(2, 1, 4, 64).contiguous()
    out = cache.attend(0, q2)
    assert torch.equal(out[0], out[1])
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    new = torch.randn((2, 1, 2, 64), device=DEV).half()
    grown, back = cache.lengths + 1, cache.lengths.clone()
    result = torch.empty_like(q2)
    with torch.cuda.graph(graph, stream=stream):
        cache.resize(grown)
        cache.append(0, new, new, back)
        cache.attend(0, q2, out=result)
        cache.resize(back)
    graph.replay()
    first = result.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert cache.device_status() == 0 and cache.lengths.tolist() == [50, 50]
    assert torch.equal(result, first)


def test_refusals():
    ralm = _ralm()
    cache, k, v, b = filled(2, 2, 64, 16, [20, 20], seed=12)
    q = torch.randn((2, 1, 4, 64), device=DEV).half()
    x = torch.randn((2, 1, 2, 64), device=DEV).half()
    for bad in (q.float(), q[..., :32], q[0], q.cpu(), q.transpose(2, 3)):
        with pytest.raises(TypeError):
            cache.attend(0, bad)
    for kwargs in (dict(q_len=i32([1])), dict(rows=i32([0, 1, 0])), dict(out=torch.empty_like(q[:1])), dict(out=q.bfloat16()),
                   dict(q_len=torch.ones(2, device=DEV, dtype=torch.int64))):
        with pytest.raises(TypeError):
            cache.attend(0, q, **kwargs)
    with pytest.raises(TypeError):
        cache.attend(0, torch.randn((3, 1, 4, 64), device=DEV).half())          # more entries than rows
    for layer, heads, scale in ((1, 4, 1.0), (-1, 4, 1.0), (0, 3, 1.0), (0, 4, float("nan"))):
        with pytest.raises(ralm.RalmError) as e:
            cache.attend(layer, torch.randn((2, 1, heads, 64), device=DEV).half(), scale=scale)
        assert e.value.status == 1
    with pytest.raises(ralm.RalmError):
        cache.attend(0, q, out=q)                                                 # in place
    for args in ((x.float(), x.float()), (x, x.bfloat16()), (x[:, :, :1], x[:, :, :1]), (x, x[:1])):
        with pytest.raises(TypeError):
            cache.append(0, *args, i32([0, 0]))
    with pytest.raises(TypeError):
        cache.append(0, x, x, i32([0]))
    with pytest.raises(TypeError):
        cache.read(0, i32([0, 0]), 2, k=x, v=x)
    for args in (dict(head_dim=96), dict(page_size=48), dict(page_size=128)):
        with pytest.raises(TypeError):
            ralm.KVCache.allocate(1, 2, args.get("head_dim", 64), 4, 2, 2, args.get("page_size", 16), device=DEV)
    assert cache.attend(0, q[:0]).shape == (0, 1, 4, 64) and cache.attend(0, q[:, :0]).shape == (2, 0, 4, 64)
