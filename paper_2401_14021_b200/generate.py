"""The generator's side of the serving loop (include/ralm.h): the KNN-LM mixture, verification of
drafted tokens, the pages of a cache, and the cache held in 4 bits with its attention.

Like binding.py this only marshals arguments: torch supplies device memory and streams."""
import ctypes

import torch

from .binding import L2, _check, _dev, _stream_ptr, load_library

_i32, _i64, _p, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
_DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}


class _Pages(ctypes.Structure):
    _fields_ = [("pool", _p), ("layers", _i64), ("layer_stride", _i64), ("page_bytes", _i64), ("pages", _i32),
                ("rows", _i32), ("max_pages", _i32), ("page_size", _i32), ("table", _p), ("lengths", _p),
                ("refs", _p), ("status", _p), ("workspace", _p)]


class _Kv(ctypes.Structure):
    _fields_ = [("pages", _Pages), ("kv_heads", _i32), ("head_dim", _i32)]


class _Tokens(ctypes.Structure):
    _fields_ = [("k", _p), ("v", _p), ("k_b", _i64), ("k_n", _i64), ("k_h", _i64), ("v_b", _i64), ("v_n", _i64),
                ("v_h", _i64), ("batch", _i32), ("n", _i32), ("dtype", _i32), ("rows", _p), ("starts", _p),
                ("count", _p)]


class _Attend(ctypes.Structure):
    _fields_ = [("q", _p), ("out", _p), ("q_b", _i64), ("q_n", _i64), ("q_h", _i64), ("o_b", _i64), ("o_n", _i64),
                ("o_h", _i64), ("batch", _i32), ("n", _i32), ("q_heads", _i32), ("dtype", _i32), ("scale", _f32),
                ("rows", _p), ("q_len", _p), ("workspace", _p), ("workspace_bytes", _i64)]


_declared = None


def _lib():
    """The library with the prototypes of this module's calls."""
    global _declared
    lib = load_library()
    if _declared is lib:
        return lib
    lib.ralm_knn_mix.argtypes = [_p, _i32, _i64, _i32, _i32, _p, _p, _i32, _i32, _p, _i64, _f32, _f32, _f32, _p, _i64, _p]
    lib.ralm_verify_tokens.argtypes = [_p, _p, _i64, _i64, _p, _i64, _i64, _p, _p, _i32, _i32, _i32, _p, _p, _p]
    lib.ralm_pages_workspace.argtypes = [_i32]
    lib.ralm_pages_workspace.restype = _i64
    lib.ralm_pages_resize.argtypes = [_p, _p, _p]
    lib.ralm_pages_fork.argtypes = [_p, _p, _p, _i32, _p]
    lib.ralm_pages_compact.argtypes = [_p, _p, _p]
    lib.ralm_pages_copy.argtypes = [_p, _p, _p, _p, _i32, _p]
    lib.ralm_pages_status.argtypes = [_p, _p]
    lib.ralm_kv_append.argtypes = [_p, _i32, _p, _p]
    lib.ralm_kv_read.argtypes = [_p, _i32, _p, _p]
    lib.ralm_kv_attend_workspace.argtypes = [_i32, _i32, _i32, _i32]
    lib.ralm_kv_attend_workspace.restype = _i64
    lib.ralm_kv_attend.argtypes = [_p, _i32, _p, _p]
    for name in ("ralm_knn_mix", "ralm_verify_tokens", "ralm_pages_resize", "ralm_pages_fork", "ralm_pages_compact",
                 "ralm_pages_copy", "ralm_pages_status", "ralm_kv_append", "ralm_kv_read", "ralm_kv_attend"):
        getattr(lib, name).restype = _i32
    _declared = lib
    return lib


def _shape(t: torch.Tensor, shape, name: str):
    if tuple(t.shape) != tuple(shape):
        raise TypeError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))


def _rows_of(t: torch.Tensor, dtypes, name: str) -> int:
    """Data pointer of a CUDA tensor whose last dimension is contiguous."""
    if not t.is_cuda or t.dtype not in dtypes or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise TypeError("%s must be a CUDA tensor of %s with a contiguous last dimension" % (name, dtypes))
    return t.data_ptr()


def _ints(t, n: int, name: str) -> int:
    if t is None:
        return 0
    _shape(t, (n,), name)
    return _dev(t, torch.int32, name)


_ANY = (torch.float16, torch.bfloat16, torch.float32)
_HALF = (torch.float16, torch.bfloat16)
_F32 = (torch.float32,)


def knn_mix(logits: torch.Tensor, ids: torch.Tensor, scores: torch.Tensor, values: torch.Tensor, lam: float,
            temperature: float = 1.0, knn_temperature: float = 1.0, metric: int = L2, probs: torch.Tensor = None,
            stream=None) -> torch.Tensor:
    """ralm_knn_mix: logits [R][V] (fp16, bf16 or fp32, any row pitch), the ids int64 [R][k] and scores
    fp32 [R][k] that `search` returned, values int32 [N] -> probs fp32 [R][V]. Without neighbours
    (ids = scores = values = None) it is softmax(logits / temperature)."""
    lib = _lib()
    R, V = logits.shape
    lp = _rows_of(logits, _ANY, "logits")
    if probs is None:
        probs = torch.empty((R, V), dtype=torch.float32, device=logits.device)
    _shape(probs, (R, V), "probs")
    pp = _rows_of(probs, _F32, "probs")
    k = N = ip = sp = vp = 0
    if ids is not None:
        k, N = ids.shape[1], values.shape[0]
        _shape(ids, (R, k), "ids")
        _shape(scores, (R, k), "scores")
        ip, sp, vp = _dev(ids, torch.int64, "ids"), _dev(scores, torch.float32, "scores"), _dev(values, torch.int32, "values")
    _check(lib.ralm_knn_mix(lp, _DTYPES[logits.dtype], logits.stride(0) if R > 1 else V, R, V, ip, sp, k, metric, vp, N,
                            lam, temperature, knn_temperature, pp, probs.stride(0) if R > 1 else V,
                            _stream_ptr(stream)), "ralm_knn_mix")
    return probs


def verify_tokens(draft_tokens: torch.Tensor, draft_probs, target_probs: torch.Tensor, uniforms: torch.Tensor,
                  draft_len: torch.Tensor = None, tokens: torch.Tensor = None, accepted: torch.Tensor = None, stream=None):
    """ralm_verify_tokens: draft_tokens int64 [R][S], draft_probs fp32 [R][S][V] or None (drafts that came
    with certainty), target_probs fp32 [R][S + 1][V], uniforms fp32 [R][S + 1], draft_len int32 [R] or
    None -> (tokens int64 [R][S + 1], accepted int32 [R])."""
    lib = _lib()
    R, S = draft_tokens.shape
    V = target_probs.shape[2]
    _shape(target_probs, (R, S + 1, V), "target_probs")
    _shape(uniforms, (R, S + 1), "uniforms")
    tp = _rows_of(target_probs, _F32, "target_probs")
    dp = d0 = d1 = 0
    if draft_probs is not None:
        _shape(draft_probs, (R, S, V), "draft_probs")
        dp, d0, d1 = _rows_of(draft_probs, _F32, "draft_probs"), draft_probs.stride(0), draft_probs.stride(1)
    if tokens is None:
        tokens = torch.empty((R, S + 1), dtype=torch.int64, device=target_probs.device)
    if accepted is None:
        accepted = torch.empty((R,), dtype=torch.int32, device=target_probs.device)
    _shape(tokens, (R, S + 1), "tokens")
    _check(lib.ralm_verify_tokens(_dev(draft_tokens, torch.int64, "draft_tokens"), dp, d0, d1, tp, target_probs.stride(0),
                                  target_probs.stride(1), _dev(uniforms, torch.float32, "uniforms"),
                                  _ints(draft_len, R, "draft_len"), R, S, V, _dev(tokens, torch.int64, "tokens"),
                                  _ints(accepted, R, "accepted"), _stream_ptr(stream)), "ralm_verify_tokens")
    return tokens, accepted


class Pages:
    """A pool of equally sized pages and the rows that hold them (ralm_pages_t). The tensors are the
    caller's: pool uint8 [layers][pages][page_bytes] (or None: bookkeeping only), table int32
    [rows][max_pages], lengths int32 [rows], refs int32 [pages]. A new pool starts from table = -1,
    lengths = refs = 0, which `Pages.allocate` makes. To be used from one stream at a time."""

    def __init__(self, pool, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor, page_size: int):
        self._lib = _lib()
        rows, max_pages = table.shape
        pages = refs.shape[0]
        _shape(lengths, (rows,), "lengths")
        self.pool, self.table, self.lengths, self.refs, self.page_size = pool, table, lengths, refs, page_size
        c = _Pages(pages=pages, rows=rows, max_pages=max_pages, page_size=page_size)
        c.table, c.lengths, c.refs = (_dev(t, torch.int32, n) for t, n in
                                      ((table, "table"), (lengths, "lengths"), (refs, "refs")))
        if pool is not None:
            if pool.dim() != 3 or pool.shape[1] != pages:
                raise TypeError("pool must be [layers][pages][page_bytes]")
            c.pool, c.layers = _dev(pool, torch.uint8, "pool"), pool.shape[0]
            c.layer_stride, c.page_bytes = pool.stride(0), pool.shape[2]
        self.status = torch.zeros(1, dtype=torch.int32, device=table.device)
        self.live = torch.zeros(1, dtype=torch.int32, device=table.device)
        self._work = torch.zeros(self._lib.ralm_pages_workspace(pages), dtype=torch.uint8, device=table.device)
        c.status, c.workspace = self.status.data_ptr(), self._work.data_ptr()
        self._c = c
        self._ptr = ctypes.addressof(c)

    @staticmethod
    def tensors(layers: int, pages: int, page_bytes: int, rows: int, max_pages: int, device="cuda"):
        """(pool, table, lengths, refs) of a pool that holds nothing yet."""
        return (torch.empty((layers, pages, page_bytes), dtype=torch.uint8, device=device),
                torch.full((rows, max_pages), -1, dtype=torch.int32, device=device),
                torch.zeros(rows, dtype=torch.int32, device=device), torch.zeros(pages, dtype=torch.int32, device=device))

    @classmethod
    def allocate(cls, layers: int, pages: int, page_bytes: int, rows: int, max_pages: int, page_size: int, device="cuda"):
        return cls(*cls.tensors(layers, pages, page_bytes, rows, max_pages, device), page_size)

    def resize(self, new_lengths: torch.Tensor, stream=None):
        """ralm_pages_resize: give back, copy on write and take pages for new_lengths int32 [rows]."""
        _check(self._lib.ralm_pages_resize(self._ptr, _ints(new_lengths, self._c.rows, "new_lengths"), _stream_ptr(stream)),
               "ralm_pages_resize")

    def fork(self, src: torch.Tensor, dst: torch.Tensor, stream=None):
        """ralm_pages_fork: rows dst int32 [n] come to hold the pages of rows src int32 [n]."""
        n = src.shape[0]
        _check(self._lib.ralm_pages_fork(self._ptr, _ints(src, n, "src"), _ints(dst, n, "dst"), n, _stream_ptr(stream)),
               "ralm_pages_fork")

    def compact(self, stream=None) -> torch.Tensor:
        """ralm_pages_compact: live pages become 0 .. live - 1; returns live, int32 [1] on the device."""
        _check(self._lib.ralm_pages_compact(self._ptr, self.live.data_ptr(), _stream_ptr(stream)), "ralm_pages_compact")
        return self.live

    def copy_from(self, other: "Pages", src: torch.Tensor, dst: torch.Tensor, stream=None):
        """ralm_pages_copy: contents of `other`'s pages src int32 [n] into this pool's pages dst int32 [n]."""
        n = src.shape[0]
        _check(self._lib.ralm_pages_copy(other._ptr, _ints(src, n, "src"), self._ptr, _ints(dst, n, "dst"), n,
                                         _stream_ptr(stream)), "ralm_pages_copy")

    def device_status(self, stream=None) -> int:
        """ralm_pages_status: reads and clears the status word (synchronises)."""
        return self._lib.ralm_pages_status(self._ptr, _stream_ptr(stream))


class KVCache(Pages):
    """A key-value cache held in 4 bits (ralm_kv_t) over a page pool of kv_heads * page_size *
    (head_dim + 8) bytes per page; head_dim 64 or 128, page_size 16, 32 or 64."""

    def __init__(self, pool: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor, *,
                 kv_heads: int, head_dim: int, page_size: int):
        if head_dim not in (64, 128) or page_size not in (16, 32, 64):
            raise TypeError("head_dim must be 64 or 128, page_size 16, 32 or 64")
        if pool is None or pool.shape[-1] != self.page_bytes(kv_heads, head_dim, page_size):
            raise TypeError("pool must have pages of %d bytes" % self.page_bytes(kv_heads, head_dim, page_size))
        super().__init__(pool, table, lengths, refs, page_size)
        self.kv_heads, self.head_dim = kv_heads, head_dim
        self._kv = _Kv(pages=self._c, kv_heads=kv_heads, head_dim=head_dim)
        self._kv_ptr = ctypes.addressof(self._kv)
        self._attend_work = {}

    @staticmethod
    def page_bytes(kv_heads: int, head_dim: int, page_size: int) -> int:
        return kv_heads * page_size * (head_dim + 8)

    @classmethod
    def allocate(cls, layers: int, kv_heads: int, head_dim: int, pages: int, rows: int, max_pages: int,
                 page_size: int = 32, device="cuda"):
        return cls(*cls.tensors(layers, pages, cls.page_bytes(kv_heads, head_dim, page_size), rows, max_pages, device),
                   kv_heads=kv_heads, head_dim=head_dim, page_size=page_size)

    def _tokens(self, k, v, starts, count, rows):
        if k.dim() != 4 or k.shape[2] != self.kv_heads or k.shape[3] != self.head_dim or k.dtype != v.dtype:
            raise TypeError("k and v must be [batch][n][%d][%d] of one type" % (self.kv_heads, self.head_dim))
        _shape(v, k.shape, "v")
        batch, n = k.shape[:2]
        if rows is None and batch > self._c.rows:
            raise TypeError("more entries than rows of the table")
        return _Tokens(_rows_of(k, _HALF, "k"), _rows_of(v, _HALF, "v"), *k.stride()[:3], *v.stride()[:3], batch, n,
                       _DTYPES[k.dtype], _ints(rows, batch, "rows"), _ints(starts, batch, "starts"),
                       _ints(count, batch, "count"))

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, count: torch.Tensor = None,
               rows: torch.Tensor = None, stream=None):
        """ralm_kv_append: k, v [batch][n][kv_heads][head_dim] (fp16 or bf16) into positions starts
        int32 [batch] and on, below the rows' lengths."""
        t = self._tokens(k, v, starts, count, rows)
        _check(self._lib.ralm_kv_append(self._kv_ptr, layer, ctypes.addressof(t), _stream_ptr(stream)), "ralm_kv_append")

    def read(self, layer: int, starts: torch.Tensor, n: int, dtype=torch.float16, k: torch.Tensor = None,
             v: torch.Tensor = None, count: torch.Tensor = None, rows: torch.Tensor = None, stream=None):
        """ralm_kv_read: the values of positions starts .. starts + n - 1 -> (k, v) [batch][n][kv_heads][head_dim]."""
        shape = (starts.shape[0], n, self.kv_heads, self.head_dim)
        if k is None:
            k = torch.empty(shape, dtype=dtype, device=starts.device)
        if v is None:
            v = torch.empty(shape, dtype=k.dtype, device=starts.device)
        _shape(k, shape, "k")
        t = self._tokens(k, v, starts, count, rows)
        _check(self._lib.ralm_kv_read(self._kv_ptr, layer, ctypes.addressof(t), _stream_ptr(stream)), "ralm_kv_read")
        return k, v

    def attend(self, layer: int, q: torch.Tensor, scale: float = None, q_len: torch.Tensor = None,
               rows: torch.Tensor = None, out: torch.Tensor = None, stream=None) -> torch.Tensor:
        """ralm_kv_attend: q [batch][n][q_heads][head_dim], the rows' newest n tokens -> out, the same shape
        and type. scale defaults to head_dim ** -0.5."""
        if q.dim() != 4 or q.shape[3] != self.head_dim:
            raise TypeError("q must be [batch][n][q_heads][%d]" % self.head_dim)
        batch, n, heads = q.shape[:3]
        if rows is None and batch > self._c.rows:
            raise TypeError("more entries than rows of the table")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        _shape(out, q.shape, "out")
        if out.dtype != q.dtype:
            raise TypeError("out must have q's type")
        work = self._attend_work.get((heads, n))
        if work is None:
            size = self._lib.ralm_kv_attend_workspace(self.kv_heads, self.head_dim, heads, n)
            work = next((w for w in self._attend_work.values() if w.numel() >= size), None)
            if work is None:
                work = torch.empty(max(size, 16), dtype=torch.uint8, device=q.device)
            self._attend_work[heads, n] = work
        a = _Attend(_rows_of(q, _HALF, "q"), _rows_of(out, _HALF, "out"), *q.stride()[:3], *out.stride()[:3], batch, n, heads,
                    _DTYPES[q.dtype], self.head_dim ** -0.5 if scale is None else scale, _ints(rows, batch, "rows"),
                    _ints(q_len, batch, "q_len"), work.data_ptr(), work.numel())
        _check(self._lib.ralm_kv_attend(self._kv_ptr, layer, ctypes.addressof(a), _stream_ptr(stream)), "ralm_kv_attend")
        return out
