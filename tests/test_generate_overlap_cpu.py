"""Outputs that overlap inputs are refused before any CUDA call, whatever the strides; what lies side by side in one buffer is
not. Without a device a call that passes its checks ends in RALM_ERR_CUDA."""
import ctypes
import itertools
import random

import pytest
import torch

OK, INVALID, CUDA = 0, 1, 3
p, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses are made up: only where no kernel can start")


@pytest.fixture(scope="module")
def lib():
    from paper_2401_14021_b200 import build
    lib = ctypes.CDLL(build.build())
    lib.ralm_knn_mix.argtypes = [p, i32, i64, i32, i32, p, p, i32, i32, p, i64, f32, f32, f32, p, i64, p]
    lib.ralm_verify_tokens.argtypes = [p, p, i64, i64, p, i64, i64, p, p, i32, i32, i32, p, p, p]
    lib.ralm_kv_attend.argtypes = [p, i32, p, p]
    lib.ralm_kv_attend_workspace.argtypes = [i32] * 4
    lib.ralm_kv_attend_workspace.restype = i64
    return lib


BASE = 1 << 32


def bytes_of(at, run, dims):
    """The set of bytes of runs of `run` bytes, dims = [(count, stride in bytes)]."""
    out = set()
    for index in itertools.product(*(range(n) for n, _ in dims)):
        first = at + sum(i * s for i, (_, s) in zip(index, dims))
        out.update(range(first, first + run))
    return out


def test_knn_mix(lib):
    def call(logits, ld, probs, ldp, R=3, V=10, dtype=2, ids=BASE << 1, scores=BASE << 2, values=BASE << 3, k=4):
        return lib.ralm_knn_mix(logits, dtype, ld, R, V, ids, scores, k, 1, values, 50, 0.5, 1.0, 1.0, probs, ldp, None)

    assert call(BASE, 10, BASE + 120, 10) == CUDA                     # one after the other
    assert call(BASE, 10, BASE + 116, 10) == INVALID                  # by one element
    assert call(BASE + 116, 10, BASE, 10) == INVALID
    assert call(BASE, 20, BASE + 40, 20) == CUDA                      # columns of one buffer
    assert call(BASE, 20, BASE + 36, 20) == INVALID
    assert call(BASE, 20, BASE + 44, 20) == INVALID                   # into the next row
    assert call(BASE, 10, BASE, 10, dtype=0) == INVALID
    far = BASE << 4
    assert call(far, 10, BASE, 10, ids=BASE + 112, k=4) == INVALID
    assert call(far, 10, BASE, 10, scores=BASE - 44) == INVALID and call(far, 10, BASE, 10, scores=BASE - 48) == CUDA
    assert call(far, 10, BASE, 10, values=BASE + 116) == INVALID and call(far, 10, BASE, 10, values=BASE + 120) == CUDA
    assert call(far, 10, BASE, 10, values=BASE, k=0) == CUDA          # not read


def test_verify_tokens(lib):
    R, S, V = 1, 4, 100
    good = dict(draft=BASE, dprobs=BASE << 1, dr=S * V, ds=V, target=BASE << 2, tr=(S + 1) * V, ts=V, u=BASE << 3, len=BASE << 4, R=R, S=S, V=V,
                tokens=BASE << 5, accepted=BASE << 6, stream=None)

    def call(**kw):
        return lib.ralm_verify_tokens(*{**good, **kw}.values())

    assert call() == CUDA
    for kw in (dict(tokens=BASE), dict(tokens=BASE + 24), dict(tokens=BASE - 32), dict(accepted=BASE << 4), dict(accepted=(BASE << 3) + 16),
               dict(accepted=(BASE << 5) + 32), dict(tokens=BASE << 2), dict(accepted=(BASE << 1) + 4 * S * V - 4), dict(accepted=BASE + 28)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(tokens=BASE + 32), dict(tokens=BASE - 40), dict(accepted=(BASE << 3) + 20), dict(accepted=(BASE << 1) + 4 * S * V),
               dict(accepted=BASE + 32), dict(len=None, accepted=BASE << 4), dict(dprobs=None, accepted=BASE << 1)):
        assert call(**kw) == CUDA, kw


class AttendArgs(ctypes.Structure):
    _fields_ = [("q", p), ("out", p)] + [(x, i64) for x in ("qb", "qn", "qh", "ob", "on", "oh")] + [
        (x, i32) for x in ("batch", "n", "q_heads", "dtype")] + [("scale", f32), ("rows", p), ("q_len", p), ("workspace", p), ("size", i64)]


def cache():
    from paper_2401_14021_b200.generate import _Kv, _Pages
    return _Kv(pages=_Pages(pool=256, layers=1, layer_stride=1152 * 16, page_bytes=1152, pages=16, rows=64, max_pages=8, page_size=16, table=256,
                            lengths=256, refs=256, status=256, workspace=256), kv_heads=1, head_dim=64)


def test_attention(lib):
    """Random layouts in one buffer against sets of bytes."""
    kv, Attend = cache(), AttendArgs
    rng = random.Random(1)
    seen = {OK: 0, INVALID: 0, CUDA: 0}
    for _ in range(3000):
        n = [rng.randint(1, 3) for _ in range(3)]
        where, sets = [], []
        for _ in range(2):
            order, strides, step = rng.sample(range(3), 3), [0] * 3, 64 + 16 * rng.choice([0, 0, 1, 4, 8])
            for d in order:                                            # nested, with gaps, in any order
                strides[d] = step
                step = step * n[d] + 16 * rng.choice([0, 0, 2, 4, 12])
            if rng.random() < 0.1:
                strides[rng.randrange(3)] = rng.choice([0, 16, 48, 80])   # steps that are not nested
            if rng.random() < 0.1:
                strides = [-x for x in strides]
            at = BASE + 32 * rng.randint(0, 40)
            where.append((at, strides))
            sets.append(bytes_of(at, 128, [(c, 2 * s) for c, s in zip(n, strides)]))
        (q, qs), (out, os_) = where
        a = Attend(q, out, *qs, *os_, *n, 0, 1.0, None, None, 256, 1 << 40)
        got = lib.ralm_kv_attend(ctypes.addressof(kv), 0, ctypes.addressof(a), None)
        assert got == (INVALID if sets[0] & sets[1] else CUDA), (n, where)
        seen[got] += 1
    assert seen[INVALID] > 300 and seen[CUDA] > 300, seen


def test_columns_of_one_buffer_are_told_apart_at_once(lib):
    """Queries, outputs and others in turn for each token, as a fused projection leaves them: however many tokens, the
    answer takes no look at each."""
    import time

    kv, Attend = cache(), AttendArgs
    took = []
    for n in (1000, 200000):
        row = 3 * 4 * 64
        for shift, want in ((4 * 64, CUDA), (4 * 64 - 8, INVALID), (2 * 4 * 64, CUDA), (row - 64, INVALID), (-4 * 64, CUDA), (-4 * 64 + 8, INVALID)):
            q = BASE << 8
            a = Attend(q, q + 2 * shift, n * row, row, 64, n * row, row, 64, 1, n, 4, 0, 1.0, None, None, 256, 1 << 60)
            begin = time.perf_counter()
            assert lib.ralm_kv_attend(ctypes.addressof(kv), 0, ctypes.addressof(a), None) == want, (n, shift)
            if want == CUDA:
                took.append(time.perf_counter() - begin)
    assert sorted(took)[len(took) // 2] < 1e-3


def test_read(lib):
    class Tokens(ctypes.Structure):
        _fields_ = [("k", p), ("v", p), ("strides", i64 * 6), ("batch", i32), ("n", i32), ("dtype", i32), ("rows", p), ("starts", p), ("count", p)]

    kv = cache()
    for call, k, v, want in ((lib.ralm_kv_read, BASE, BASE, INVALID), (lib.ralm_kv_read, BASE, BASE + 120, INVALID),
                             (lib.ralm_kv_read, BASE, BASE + 128, CUDA), (lib.ralm_kv_append, BASE, BASE, CUDA)):
        t = Tokens(k, v, (i64 * 6)(1280, 128, 64, 1280, 128, 64), 3, 10, 0, None, 256, None)
        call.argtypes = [p, i32, p, p]
        assert call(ctypes.addressof(kv), 0, ctypes.addressof(t), None) == want
