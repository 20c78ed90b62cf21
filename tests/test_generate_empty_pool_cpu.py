"""A cache over a pool without pages: where a length promises tokens there is no page that attention could read instead of a
bad one, so the calls refuse the pool before any CUDA call."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses are made up: only where no kernel can start")


def test_a_pool_without_pages_is_refused():
    from paper_2401_14021_b200 import build
    from paper_2401_14021_b200.generate import _Kv, _Pages
    lib = ctypes.CDLL(build.build())
    p, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64

    class Attend(ctypes.Structure):
        _fields_ = [("q", p), ("out", p), ("strides", i64 * 6), ("batch", i32), ("n", i32), ("q_heads", i32), ("dtype", i32),
                    ("scale", ctypes.c_float), ("rows", p), ("q_len", p), ("workspace", p), ("size", i64)]

    class Tokens(ctypes.Structure):
        _fields_ = [("k", p), ("v", p), ("strides", i64 * 6), ("batch", i32), ("n", i32), ("dtype", i32), ("rows", p), ("starts", p), ("count", p)]

    attend = Attend(1 << 20, 1 << 21, (i64 * 6)(*[64] * 6), 1, 1, 1, 0, 1.0, None, None, 256, 1 << 40)
    tokens = Tokens(1 << 20, 1 << 21, (i64 * 6)(*[64] * 6), 1, 1, 0, None, 256, None)
    for pages, want in ((0, 1), (1, 3)):          # RALM_ERR_INVALID_ARG; with a page the checks pass and the device is missing
        kv = _Kv(pages=_Pages(pool=256, layers=1, layer_stride=1152 * 16, page_bytes=1152, pages=pages, rows=4, max_pages=8, page_size=16,
                              table=256, lengths=256, refs=256, status=256, workspace=256), kv_heads=1, head_dim=64)
        for call, what in ((lib.ralm_kv_attend, attend), (lib.ralm_kv_append, tokens), (lib.ralm_kv_read, tokens)):
            call.argtypes = [p, i32, p, p]
            assert call(ctypes.addressof(kv), 0, ctypes.addressof(what), None) == want, (call, pages)
