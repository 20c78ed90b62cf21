"""The generator's side of the serving loop (include/ralm.h): the KNN-LM mixture, verification of
drafted tokens, the pages of a cache, and the cache held in 4 bits with its attention.

Like binding.py this only marshals arguments (in csrc/binding.cpp, where the checks of a call cost less
than a kernel launch): torch supplies device memory and streams."""
import ctypes
import os

import torch

from .binding import L2, RalmError, _dev, _stream_ptr, load_library

_i32, _i64, _p = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class _Pages(ctypes.Structure):
    _fields_ = [("pool", _p), ("layers", _i64), ("layer_stride", _i64), ("page_bytes", _i64), ("pages", _i32),
                ("rows", _i32), ("max_pages", _i32), ("page_size", _i32), ("table", _p), ("lengths", _p),
                ("refs", _p), ("status", _p), ("workspace", _p)]


class _Kv(ctypes.Structure):
    _fields_ = [("pages", _Pages), ("kv_heads", _i32), ("head_dim", _i32)]


_calls = None


def _native():
    """The marshalling module, holding the entry points of the loaded library."""
    global _calls
    lib = load_library()
    if _calls is not None and _calls[0] is lib:
        return _calls[1]
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_native.so")
    if not os.path.exists(path):
        raise RuntimeError("%s is missing: build it with `python -m paper_2401_14021_b200.build`" % path)
    from . import _native as module
    names = ("ralm_knn_mix", "ralm_verify_tokens", "ralm_pages_resize", "ralm_pages_fork", "ralm_pages_compact",
             "ralm_pages_copy", "ralm_kv_append", "ralm_kv_read", "ralm_kv_attend")
    module.bind({name: ctypes.cast(getattr(lib, name), _p).value for name in names}, RalmError)
    lib.ralm_pages_workspace.argtypes = [_i32]
    lib.ralm_pages_workspace.restype = _i64
    lib.ralm_pages_status.argtypes = [_p, _p]
    lib.ralm_pages_status.restype = _i32
    lib.ralm_kv_attend_workspace.argtypes = [_i32, _i32, _i32, _i32]
    lib.ralm_kv_attend_workspace.restype = _i64
    _calls = (lib, module)
    return module


def knn_mix(logits: torch.Tensor, ids: torch.Tensor, scores: torch.Tensor, values: torch.Tensor, lam: float,
            temperature: float = 1.0, knn_temperature: float = 1.0, metric: int = L2, probs: torch.Tensor = None,
            stream=None) -> torch.Tensor:
    """ralm_knn_mix: logits [R][V] (fp16, bf16 or fp32, any row pitch), the ids int64 [R][k] and scores
    fp32 [R][k] that `search` returned, values int32 [N] -> probs fp32 [R][V]. Without neighbours
    (ids = scores = values = None) it is softmax(logits / temperature)."""
    return (_calls[1] if _calls else _native()).knn_mix(logits, ids, scores, values, lam, temperature, knn_temperature,
                                                        metric, probs, stream)


def verify_tokens(draft_tokens: torch.Tensor, draft_probs, target_probs: torch.Tensor, uniforms: torch.Tensor,
                  draft_len: torch.Tensor = None, tokens: torch.Tensor = None, accepted: torch.Tensor = None, stream=None):
    """ralm_verify_tokens: draft_tokens int64 [R][S], draft_probs fp32 [R][S][V] or None (drafts that came
    with certainty), target_probs fp32 [R][S + 1][V], uniforms fp32 [R][S + 1], draft_len int32 [R] or
    None -> (tokens int64 [R][S + 1], accepted int32 [R])."""
    return (_calls[1] if _calls else _native()).verify_tokens(draft_tokens, draft_probs, target_probs, uniforms,
                                                              draft_len, tokens, accepted, stream)


def _shape(t: torch.Tensor, shape, name: str):
    if tuple(t.shape) != tuple(shape):
        raise TypeError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))


class Pages:
    """A pool of equally sized pages and the rows that hold them (ralm_pages_t). The tensors are the
    caller's: pool uint8 [layers][pages][page_bytes] (or None: bookkeeping only), table int32
    [rows][max_pages], lengths int32 [rows], refs int32 [pages]. A new pool starts from table = -1,
    lengths = refs = 0, which `Pages.allocate` makes. To be used from one stream at a time."""

    def __init__(self, pool, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor, page_size: int):
        self._call = _native()
        self._lib = load_library()
        rows, max_pages = table.shape
        pages = refs.shape[0]
        _shape(lengths, (rows,), "lengths")
        if any(t is not None and t.device != table.device for t in (pool, lengths, refs)):
            raise TypeError("pool, table, lengths and refs must be on one device")
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
        self._call.pages_resize(self._ptr, self.table, new_lengths, stream)

    def fork(self, src: torch.Tensor, dst: torch.Tensor, stream=None):
        """ralm_pages_fork: rows dst int32 [n] come to hold the pages of rows src int32 [n]."""
        self._call.pages_fork(self._ptr, self.table, src, dst, stream)

    def compact(self, stream=None) -> torch.Tensor:
        """ralm_pages_compact: live pages become 0 .. live - 1; returns live, int32 [1] on the device."""
        return self._call.pages_compact(self._ptr, self.live, stream)

    def copy_from(self, other: "Pages", src: torch.Tensor, dst: torch.Tensor, stream=None):
        """ralm_pages_copy: contents of `other`'s pages src int32 [n] into this pool's pages dst int32 [n]."""
        self._call.pages_copy(other._ptr, src, self._ptr, dst, self.table, other.table, stream)

    def device_status(self, stream=None) -> int:
        """ralm_pages_status: reads and clears the status word (synchronises `stream`, or the current stream of the
        pool's device)."""
        with torch.cuda.device(self.table.device):
            return self._lib.ralm_pages_status(self._ptr, _stream_ptr(stream))


class KVCache(Pages):
    """A key-value cache held in 4 bits (ralm_kv_t) over a page pool of kv_heads * page_size *
    (head_dim + 8) bytes per page; head_dim 64 or 128, page_size 16, 32 or 64. Attention's workspace (23 MB for head_dim 64, 46 MB for 128) is
    made and cleared here, on the current stream; a call on another one comes after that, as with any tensor."""

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
        self._scale = head_dim ** -0.5
        with torch.cuda.device(table.device):     # room for the partial results of split rows, whatever a call's sizes
            size = max(self._lib.ralm_kv_attend_workspace(kv_heads, head_dim, kv_heads, n) for n in (8, 16, 24, 32))
            self._attend_work = torch.zeros(size, dtype=torch.uint8, device=table.device)

    @staticmethod
    def page_bytes(kv_heads: int, head_dim: int, page_size: int) -> int:
        return kv_heads * page_size * (head_dim + 8)

    @classmethod
    def allocate(cls, layers: int, kv_heads: int, head_dim: int, pages: int, rows: int, max_pages: int,
                 page_size: int = 32, device="cuda"):
        return cls(*cls.tensors(layers, pages, cls.page_bytes(kv_heads, head_dim, page_size), rows, max_pages, device),
                   kv_heads=kv_heads, head_dim=head_dim, page_size=page_size)

    def device_status(self, stream=None) -> int:
        status = super().device_status(stream)
        if status == 4:                                  # RALM_ERR_TIMEOUT: an attention call did not finish
            with torch.cuda.device(self.table.device), torch.cuda.stream(stream):
                self._attend_work.zero_()
        return status

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, count: torch.Tensor = None,
               rows: torch.Tensor = None, stream=None):
        """ralm_kv_append: k, v [batch][n][kv_heads][head_dim] (fp16 or bf16) into positions starts
        int32 [batch] and on, below the rows' lengths."""
        self._call.kv_append(self._kv_ptr, layer, k, v, starts, count, rows, stream, self.table)

    def read(self, layer: int, starts: torch.Tensor, n: int, dtype=torch.float16, k: torch.Tensor = None,
             v: torch.Tensor = None, count: torch.Tensor = None, rows: torch.Tensor = None, stream=None):
        """ralm_kv_read: the values of positions starts .. starts + n - 1 -> (k, v) [batch][n][kv_heads][head_dim], of
        k's type where one is given."""
        return self._call.kv_read(self._kv_ptr, layer, k, v, starts, count, rows, stream, self.table, n, dtype)

    def attend(self, layer: int, q: torch.Tensor, scale: float = None, q_len: torch.Tensor = None,
               rows: torch.Tensor = None, out: torch.Tensor = None, stream=None) -> torch.Tensor:
        """ralm_kv_attend: q [batch][n][q_heads][head_dim], the rows' newest n tokens -> out, the same shape
        and type. scale defaults to head_dim ** -0.5."""
        return self._call.kv_attend(self._kv_ptr, layer, q, self._scale if scale is None else scale, q_len, rows, out,
                                    self._attend_work, stream)
