"""Host-side checks of the generator's entry points: refusals come before any CUDA call."""
import ctypes

import pytest
import torch

INVALID, UNSUPPORTED = 1, 5


@pytest.fixture(scope="module")
def lib():
    from paper_2401_14021_b200 import build
    return ctypes.CDLL(build.build())


def test_knn_mix_arguments(lib):
    p, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.ralm_knn_mix.argtypes = [p, i32, i64, i32, i32, p, p, i32, i32, p, i64, f32, f32, f32, p, i64, p]
    good = dict(logits=16, dtype=0, ld=100, R=2, V=100, ids=16, scores=16, k=4, metric=1, values=16, N=10, lam=0.5, T=1.0,
                tau=1.0, probs=16, ldp=100, stream=None)

    def call(**kw):
        return lib.ralm_knn_mix(*{**good, **kw}.values())

    inf = float("inf")
    for bad in (dict(logits=None), dict(probs=None), dict(ids=None), dict(scores=None), dict(values=None), dict(R=-1), dict(V=0),
                dict(V=(1 << 22) + 1, ld=1 << 23, ldp=1 << 23), dict(ld=99), dict(ldp=99), dict(k=-1), dict(k=1025), dict(N=-1),
                dict(dtype=3), dict(metric=2), dict(lam=-0.01), dict(lam=1.01), dict(lam=float("nan")), dict(T=0.0), dict(T=inf),
                dict(tau=-1.0), dict(tau=float("nan")), dict(logits=17)):
        assert call(**bad) == INVALID, bad
    assert call(R=0, logits=None, probs=None) == 0


def test_verify_tokens_arguments(lib):
    p, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.ralm_verify_tokens.argtypes = [p, p, i64, i64, p, i64, i64, p, p, i32, i32, i32, p, p, p]
    good = [16, None, 0, 0, 16, 100, 100, 16, None, 2, 3, 100, 16, 16, None]
    for at, value in ((0, None), (4, None), (7, None), (9, -1), (10, -1), (11, 0), (11, (1 << 22) + 1), (12, None), (13, None)):
        args = list(good)
        args[at] = value
        assert lib.ralm_verify_tokens(*args) == INVALID, at
    args = list(good)
    args[9] = 0
    assert lib.ralm_verify_tokens(*args) == 0


def test_pages_and_cache_arguments(lib):
    from paper_2401_14021_b200.generate import _Kv, _Pages
    p, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.ralm_pages_workspace.restype = i64
    lib.ralm_pages_workspace.argtypes = [i32]
    assert lib.ralm_pages_workspace(-1) == 0 and lib.ralm_pages_workspace(10) > 0
    good = dict(pool=256, layers=2, layer_stride=16 * 1152 * 4, page_bytes=1152, pages=16, rows=4, max_pages=8, page_size=16,
                table=256, lengths=256, refs=256, status=256, workspace=256)
    for name in ("ralm_pages_resize", "ralm_pages_fork", "ralm_pages_compact"):
        getattr(lib, name).argtypes = [p, p, p] if name != "ralm_pages_fork" else [p, p, p, i32, p]

    for bad in (dict(table=None), dict(lengths=None), dict(refs=None), dict(status=None), dict(workspace=None), dict(pages=-1),
                dict(rows=-1), dict(rows=65537), dict(max_pages=0), dict(max_pages=(1 << 20) + 1), dict(page_size=0),
                dict(max_pages=1 << 20, page_size=1 << 12), dict(pool=264), dict(page_bytes=1160), dict(layers=0),
                dict(layer_stride=1152), dict(layer_stride=16 * 1152 + 8)):
        c = _Pages(**{**good, **bad})
        assert lib.ralm_pages_resize(ctypes.addressof(c), 256, None) == INVALID, bad
        assert lib.ralm_pages_compact(ctypes.addressof(c), 256, None) == INVALID, bad
    c = _Pages(**good)
    assert lib.ralm_pages_resize(ctypes.addressof(c), None, None) == INVALID
    assert lib.ralm_pages_resize(None, 256, None) == INVALID
    assert lib.ralm_pages_compact(ctypes.addressof(c), None, None) == INVALID
    assert lib.ralm_pages_fork(ctypes.addressof(c), 256, 256, -1, None) == INVALID
    assert lib.ralm_pages_fork(ctypes.addressof(c), 256, 256, 5, None) == INVALID      # more pairs than rows
    assert lib.ralm_pages_fork(ctypes.addressof(c), None, 256, 2, None) == INVALID
    assert lib.ralm_pages_fork(ctypes.addressof(c), None, None, 0, None) == 0

    # the 4-bit cache: 1 head of 64 dimensions, pages of 16 tokens are 1152 bytes
    lib.ralm_kv_attend_workspace.restype = i64
    lib.ralm_kv_attend_workspace.argtypes = [i32] * 4
    for bad in ((0, 64, 4, 1), (2, 64, 3, 1), (2, 96, 4, 1), (2, 64, 4, -1), (4, 64, 2, 1)):
        assert lib.ralm_kv_attend_workspace(*bad) == 0, bad
    assert lib.ralm_kv_attend_workspace(2, 64, 4, 0) >= 0                              # no queries: no division by them
    lib.ralm_kv_attend.argtypes = lib.ralm_kv_append.argtypes = lib.ralm_kv_read.argtypes = [p, i32, p, p]
    for bad in (dict(kv_heads=0), dict(kv_heads=2), dict(head_dim=65)):
        kv = _Kv(pages=_Pages(**good), **{"kv_heads": 1, "head_dim": 64, **bad})
        for call in (lib.ralm_kv_attend, lib.ralm_kv_append, lib.ralm_kv_read):
            assert call(ctypes.addressof(kv), 0, None, None) == INVALID, bad
    kv = _Kv(pages=_Pages(**good), kv_heads=1, head_dim=64)
    for layer in (-1, 2):
        assert lib.ralm_kv_append(ctypes.addressof(kv), layer, None, None) == INVALID


def test_tensors_on_the_cpu_are_refused():
    import paper_2401_14021_b200 as ralm
    x = torch.zeros((2, 8))
    with pytest.raises(TypeError):
        ralm.knn_mix(x, None, None, None, 0.5)
    with pytest.raises(TypeError):
        ralm.verify_tokens(torch.zeros((2, 1), dtype=torch.int64), None, torch.zeros((2, 2, 8)), torch.zeros((2, 2)))
    with pytest.raises(TypeError):
        ralm.knn_mix("logits", None, None, None, 0.5)


def test_marshalling_fails_loudly_when_it_is_missing(monkeypatch, tmp_path):
    from paper_2401_14021_b200 import generate
    monkeypatch.setattr(generate, "_calls", None)
    monkeypatch.setattr(generate, "__file__", str(tmp_path / "generate.py"))
    with pytest.raises(RuntimeError):
        generate.knn_mix(torch.zeros((1, 1)), None, None, None, 0.5)
