"""Thin ctypes binding of the paged 4-bit cache (the entry points shotkv_kv4_*, shotkv_pages_* and shotkv_qk_norm_rope of
include/shotkv.h).  Argument marshalling only, as in `shotkv`; nothing here synchronises.

Rows are tensors [T, heads, D] or [P, N, heads, D] (T = P * N tokens) of any strides whose last dimension is dense and whose
rows start at multiples of 16 bytes: a cache [P, H_kv, N, D] is passed as `k.transpose(1, 2)`, a slice of a fused projection
as it is.
"""
from __future__ import annotations

import ctypes
import dataclasses
import functools

import torch

from . import shotkv
from .shotkv import ShotKVError, _check, _dtype_code, _ptr

ST_OK, ST_NO_FREE_PAGE, ST_BAD_LENGTH = 0, -4, -5
_I32, _U8, _F32 = torch.int32, torch.uint8, torch.float32


class _Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("seq_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("seq_tokens", ctypes.c_int32)]


class _Rope(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("n_positions", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("eps", ctypes.c_float), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p)]


_lib = None


def load_library() -> ctypes.CDLL:
    """libshotkv.so with the prototypes of this module's entry points declared."""
    global _lib
    if _lib is None:
        lib = shotkv.load_library()
        vp, i32, sz, cfg = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.POINTER(shotkv._Config)
        rows, cache, rope = ctypes.POINTER(_Rows), ctypes.POINTER(_Cache), ctypes.POINTER(_Rope)
        lib.shotkv_kv4_page_bytes.restype = sz
        lib.shotkv_kv4_page_bytes.argtypes = [i32, i32, i32]
        lib.shotkv_pages_plan.argtypes = [i32] * 3 + [vp] * 4 + [i32] + [vp] * 5 + [i32, i32, vp, vp, vp, vp]
        lib.shotkv_pages_release.argtypes = [i32, i32, i32, vp, vp, vp, vp, i32, vp, vp]
        lib.shotkv_qk_norm_rope.argtypes = [cfg, i32, rope, vp, rows, rows, rows, rows, rows, cache, vp, vp]
        lib.shotkv_kv4_store.argtypes = [cfg, i32, rows, rows, cache, vp, vp]
        lib.shotkv_kv4_load.argtypes = [cfg, i32, cache, vp, rows, rows, vp]
        lib.shotkv_kv4_attention_workspace_bytes.restype = sz
        lib.shotkv_kv4_attention_workspace_bytes.argtypes = [cfg, i32, i32, i32, i32, i32]
        lib.shotkv_kv4_attention.argtypes = [cfg, i32, i32, i32, cache, vp, i32, vp, vp, rows, rows, vp, vp, sz, vp]
        for name in ("pages_plan", "pages_release", "qk_norm_rope", "kv4_store", "kv4_load", "kv4_attention"):
            getattr(lib, "shotkv_" + name).restype = ctypes.c_int
        _lib = lib
    return _lib


def _stream():
    """The current stream's handle.  Without the stream object that torch.cuda.current_stream() makes (2.7 us), where torch has
    the names for that: a call for one token is a few microseconds in all."""
    return _raw_stream(_device())


# names that torch keeps to itself, and has in builds for GPUs only
_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
if _raw_stream is None or _device is None:
    _stream = shotkv._stream


def _array(t, dtype, shape, name):
    """Address of a dense GPU tensor; what is wrong with one is said by shotkv's _ptr."""
    if t is not None and t.dtype is dtype and t.is_cuda and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    return _ptr(t, dtype, shape, name)


def _dense(t, dtype, name):
    """The same for any shape."""
    if t.dtype is dtype and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    return _ptr(t, dtype, None, name)


@functools.lru_cache(maxsize=64)
def _heads(n_q_heads, n_kv_heads, head_dim, dtype, sm_scale=1.0):
    return shotkv._Config(n_q_heads, n_kv_heads, head_dim, 1, _dtype_code(dtype), sm_scale, shotkv.SELECT_PREFIX,
                          shotkv.HEADS_PER_LAYER, None)


def _rows(t, heads, D, dtype, tokens, name):
    """The shotkv_rows of a tensor [T, heads, D] or [P, N, heads, D].  (Strides of dimensions of one may be anything.)"""
    shape, stride = t.shape, t.stride()
    if t.dtype is dtype and t.is_cuda and stride[-1] == 1:
        if shape == (tokens, heads, D):
            return _Rows(t.data_ptr(), 0, stride[0] if tokens > 1 else 0, stride[1] if heads > 1 else 0, tokens or 1)
        if len(shape) == 4 and shape[2:] == (heads, D) and shape[0] * shape[1] == tokens:
            return _Rows(t.data_ptr(), stride[0] if shape[0] > 1 else 0, stride[1] if shape[1] > 1 else 0,
                         stride[2] if heads > 1 else 0, shape[1] or 1)
    if not t.is_cuda:
        raise ShotKVError(f"{name} must live on the GPU")
    if t.dtype != dtype:
        raise ShotKVError(f"{name} must be {dtype}, got {t.dtype}")
    if len(shape) not in (3, 4) or shape[-2] != heads or shape[-1] != D:
        raise ShotKVError(f"{name} must have shape (tokens, {heads}, {D}) or (P, N, {heads}, {D}), got {tuple(shape)}")
    if stride[-1] != 1:
        raise ShotKVError(f"{name} must have a dense last dimension")
    raise ShotKVError(f"{name} must have {tokens} tokens, got shape {tuple(shape)}")


def _token_rows(t):
    """Tokens, heads and D of a tensor [T, heads, D] or [P, N, heads, D]."""
    shape = t.shape
    if len(shape) == 3:
        return shape
    if len(shape) != 4:
        raise ShotKVError(f"rows must have shape (tokens, heads, D) or (P, N, heads, D), got {tuple(shape)}")
    return shape[0] * shape[1], shape[2], shape[3]


def page_bytes(page_size: int, n_kv_heads: int, head_dim: int) -> int:
    n = load_library().shotkv_kv4_page_bytes(page_size, n_kv_heads, head_dim)
    if n == 0:
        raise ShotKVError("unsupported shape of a page")
    return int(n)


class Cache:
    """A pool of pages [n_pages, page_bytes] uint8 (or any shape of as many bytes) and its geometry.  Every call looks at the
    pages as they are then: their memory, their number and the tensor itself may change between calls."""

    def __init__(self, pages, page_size, n_kv_heads, head_dim):
        self.pages, self.page_size, self.n_kv_heads, self.head_dim = pages, page_size, n_kv_heads, head_dim
        self._page_bytes = page_bytes(page_size, n_kv_heads, head_dim)
        self.c  # (checks the pages)

    @property
    def n_pages(self):
        return self.pages.numel() // self._page_bytes

    @property
    def c(self):
        """The shotkv_kv4_cache of a call."""
        pages = self.pages
        ptr = _dense(pages, _U8, "pages")
        n_pages, rest = divmod(pages.numel(), self._page_bytes)
        if rest or not n_pages:
            raise ShotKVError(f"pages must hold a whole number of pages of {self._page_bytes} bytes, got {pages.numel()} bytes")
        return _Cache(ptr, n_pages, self.page_size)

    @classmethod
    def empty(cls, n_pages, page_size, n_kv_heads, head_dim, device="cuda"):
        size = page_bytes(page_size, n_kv_heads, head_dim)
        return cls(torch.empty((n_pages, size), dtype=torch.uint8, device=device), page_size, n_kv_heads, head_dim)

    def _cfg(self, n_q_heads, dtype, sm_scale=1.0):
        return _heads(n_q_heads, self.n_kv_heads, self.head_dim, dtype, sm_scale)


@dataclasses.dataclass
class PagePlan:
    block_table: torch.Tensor   # [R, max_pages] int32, updated in place
    free_left: torch.Tensor     # [1] int32
    seq_lens: torch.Tensor      # [R] int32
    query_start: torch.Tensor   # [R + 1] int32
    slot_map: torch.Tensor      # [T] int32
    token_pos: torch.Tensor     # [T] int32
    status: torch.Tensor        # [R] int32

    def addresses(self):
        """R, max_pages, T and the tensors' addresses as they are now."""
        R, max_pages = self.block_table.shape
        T = self.slot_map.shape[0]
        one, requests, tokens = (1,), (R,), (T,)
        return (R, max_pages, T, _array(self.block_table, _I32, (R, max_pages), "block_table"), _array(self.free_left, _I32, one, "free_left"),
                _array(self.seq_lens, _I32, requests, "seq_lens"), _array(self.query_start, _I32, (R + 1,), "query_start"),
                _array(self.slot_map, _I32, tokens, "slot_map"), _array(self.token_pos, _I32, tokens, "token_pos"),
                _array(self.status, _I32, requests, "status"))

    @classmethod
    def empty(cls, block_table, tokens):
        """Buffers for plans of up to `tokens` new tokens over a block table of the caller's."""
        R, dev = block_table.shape[0], block_table.device
        make = lambda n: torch.empty(n, dtype=torch.int32, device=dev)  # noqa: E731
        return cls(block_table, make(1), make(R), make(R + 1), make(tokens), make(tokens), make(R))


def pages_plan(page_size, cached_lens, new_lens, free_pages, free_count, plan: PagePlan, pos_start=None, request_tokens=0):
    """shotkv_pages_plan.  cached_lens, new_lens [R] int32, free_pages int32 (the stack), free_count [1] int32; results go
    into `plan` (its block table is updated).  free_left and seq_lens must not be free_count and cached_lens: a loop copies them
    there for the next plan.  With request_tokens the batch is of equal shares, for `store`; `attention` takes batches without
    gaps, which plan.query_start is of."""
    R, max_pages, T, table, free_left, seq_lens, query_start, slot_map, token_pos, status = plan.addresses()
    rc = load_library().shotkv_pages_plan(
        R, page_size, max_pages, _array(cached_lens, _I32, (R,), "cached_lens"), _array(new_lens, _I32, (R,), "new_lens"),
        None if pos_start is None else _array(pos_start, _I32, (R,), "pos_start"), _dense(free_pages, _I32, "free_pages"),
        free_pages.numel(), _array(free_count, _I32, (1,), "free_count"), table, free_left, seq_lens, query_start, T, request_tokens, slot_map,
        token_pos, status, _stream())
    if rc:
        _check(rc, "shotkv_pages_plan")
    return plan


def pages_release(page_size, finished, seq_lens, block_table, free_pages, free_count):
    """shotkv_pages_release: seq_lens, block_table, free_pages and free_count are updated in place.  Every entry of a finished
    request's pages goes onto the stack that is not negative: put -1 in the place of pages that other requests still use."""
    R, max_pages = block_table.shape
    rc = load_library().shotkv_pages_release(
        R, page_size, max_pages, _array(finished, _U8, (R,), "finished"), _array(seq_lens, _I32, (R,), "seq_lens"),
        _array(block_table, _I32, (R, max_pages), "block_table"), _dense(free_pages, _I32, "free_pages"), free_pages.numel(),
        _array(free_count, _I32, (1,), "free_count"), _stream())
    if rc:
        _check(rc, "shotkv_pages_release")


class Rope:
    """Rotation and norms of qk_norm_rope: table [n_positions, rot_dim] float32 (cosines, then sines), weights [D] of the
    rows' dtype or None.  Every call looks at the tensors as they are then."""

    def __init__(self, table, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
        self.table, self.q_weight, self.k_weight, self.eps, self.interleaved = table, q_weight, k_weight, eps, interleaved
        if q_weight is not None and k_weight is not None and (q_weight.dtype, q_weight.shape) != (k_weight.dtype, k_weight.shape):
            raise ShotKVError(f"k_weight must be {q_weight.dtype} of shape {tuple(q_weight.shape)}, got {k_weight.dtype} of {tuple(k_weight.shape)}")
        self.of_rows()

    def of_rows(self, dtype=None, D=None):
        """The shotkv_rope of a call with rows of D elements of a type (None: of whatever the weights are for)."""
        table, q, k, shape = self.table, self.q_weight, self.k_weight, self.table.shape
        if len(shape) != 2:
            raise ShotKVError("table must have shape (n_positions, rot_dim)")
        of = None if dtype is None else (D,)
        if q is not None:
            q = _array(q, dtype, of, "q_weight")
        if k is not None:
            k = _array(k, dtype, of, "k_weight")
        return _Rope(_dense(table, _F32, "table"), shape[0], shape[1], 1 if self.interleaved else 0, self.eps, q, k)

    @property
    def c(self):
        return self.of_rows()


def qk_norm_rope(rope: Rope, q, k, token_pos, q_out=None, k_out=None, v=None, cache: Cache | None = None, slot_map=None):
    """shotkv_qk_norm_rope.  q, q_out rows of n_q_heads, k, k_out, v rows of n_kv_heads, token_pos and slot_map [T] int32.
    q_out, and k_out where there is no cache, are made if not given.  Returns (q_out, k_out)."""
    T, H, D = _token_rows(q)
    Hkv, dtype = k.shape[-2], q.dtype
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=dtype, device=q.device)
    if k_out is None and cache is None:
        k_out = torch.empty(k.shape, dtype=dtype, device=k.device)
    if cache is not None and (cache.n_kv_heads != Hkv or cache.head_dim != D):
        raise ShotKVError(f"the cache has rows of ({cache.n_kv_heads}, {cache.head_dim}), the keys of ({Hkv}, {D})")
    rc = load_library().shotkv_qk_norm_rope(
        _heads(H, Hkv, D, dtype), T, rope.of_rows(dtype, D), _array(token_pos, _I32, (T,), "token_pos"), _rows(q, H, D, dtype, T, "q"),
        _rows(k, Hkv, D, dtype, T, "k"), _rows(q_out, H, D, dtype, T, "q_out"),
        None if k_out is None else _rows(k_out, Hkv, D, dtype, T, "k_out"), None if v is None else _rows(v, Hkv, D, dtype, T, "v"),
        None if cache is None else cache.c, None if slot_map is None else _array(slot_map, _I32, (T,), "slot_map"), _stream())
    if rc:
        _check(rc, "shotkv_qk_norm_rope")
    return q_out, k_out


def store(cache: Cache, k, v, slot_map):
    """shotkv_kv4_store: rows of keys and values into their slots [T] int32."""
    T, H, D, dtype = _token_rows(k)[0], cache.n_kv_heads, cache.head_dim, k.dtype
    rc = load_library().shotkv_kv4_store(
        cache._cfg(H, dtype), T, _rows(k, H, D, dtype, T, "k"), _rows(v, H, D, dtype, T, "v"), cache.c, _array(slot_map, _I32, (T,), "slot_map"),
        _stream())
    if rc:
        _check(rc, "shotkv_kv4_store")


def load(cache: Cache, slot_map, k_out=None, v_out=None, dtype=torch.bfloat16):
    """shotkv_kv4_load: the rows of slots [T] int32, zeros where a slot is none.  Returns (k_out, v_out)."""
    T, H, D = slot_map.shape[0], cache.n_kv_heads, cache.head_dim
    k_out = torch.empty((T, H, D), dtype=dtype, device=slot_map.device) if k_out is None else k_out
    v_out = torch.empty((T, H, D), dtype=k_out.dtype, device=slot_map.device) if v_out is None else v_out
    dtype = k_out.dtype
    rc = load_library().shotkv_kv4_load(
        cache._cfg(H, dtype), T, cache.c, _array(slot_map, _I32, (T,), "slot_map"),
        _rows(k_out, H, D, dtype, T, "k_out"), _rows(v_out, H, D, dtype, T, "v_out"), _stream())
    if rc:
        _check(rc, "shotkv_kv4_load")
    return k_out, v_out


def attention_workspace(cache: Cache, q, block_table, max_q_len=1):
    """A workspace for attention() calls with these shapes: queries of as many tokens, a table of as many requests and pages."""
    R, max_pages = block_table.shape
    n = load_library().shotkv_kv4_attention_workspace_bytes(cache._cfg(q.shape[-2], q.dtype), R, _token_rows(q)[0],
                                                            max_q_len, cache.page_size, max_pages)
    if n == 0:
        raise ShotKVError("unsupported attention shape")
    return torch.empty(int(n), dtype=torch.uint8, device=q.device)


def attention(cache: Cache, q, block_table, seq_lens, sm_scale, query_start=None, max_q_len=None, out=None, lse=None,
              workspace=None):
    """shotkv_kv4_attention.  q rows of n_q_heads, block_table [R, max_pages], seq_lens [R], query_start [R + 1] int32 (None:
    one token per request), max_q_len the most new tokens of a request (None: as many as there are; a smaller bound takes less
    workspace and often less time), lse [T, n_q_heads] float32 or None.  Returns out; rows of tokens that no request has are
    zeros if it is made here, and stay as they are in tensors of the caller's."""
    T, H, _ = _token_rows(q)
    D, dtype = cache.head_dim, q.dtype
    R, max_pages = block_table.shape
    if max_q_len is None:
        max_q_len = 1 if query_start is None else max(T, 1)
    if out is None:
        out = (torch.empty if query_start is None else torch.zeros)(q.shape, dtype=dtype, device=q.device)
    if workspace is None:
        workspace = attention_workspace(cache, q, block_table, max_q_len)
    rc = load_library().shotkv_kv4_attention(
        cache._cfg(H, dtype, sm_scale), R, T, max_q_len, cache.c, _array(block_table, _I32, (R, max_pages), "block_table"),
        max_pages, _array(seq_lens, _I32, (R,), "seq_lens"),
        None if query_start is None else _array(query_start, _I32, (R + 1,), "query_start"),
        _rows(q, H, D, dtype, T, "q"), _rows(out, H, D, dtype, T, "out"),
        None if lse is None else _array(lse, _F32, (T, H), "lse"), _array(workspace, _U8, workspace.shape, "workspace"), workspace.numel(),
        _stream())
    if rc:
        _check(rc, "shotkv_kv4_attention")
    return out
