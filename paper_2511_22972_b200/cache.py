"""Paged key/value cache and the attention of a chunk of new tokens over it: binding of include/fly_cache.h.

Argument marshalling only, as in `binding`: the work runs in the CUDA kernels of libfly_verify.so, and the calls of every
step are marshalled by the native extension.  One round of a layer:

    cache_append(cache, k, v, stream=st)                 # [B, K+1, kv_heads, head_dim] behind cache.lengths
    attention.run(cache, q, out, stream=st)              # [B, K+1, heads, head_dim]
    ...                                                  # the last layer's hidden states: verify_fused
    cache.lengths.add_(buffers.accept_len).sub_(buffers.rollback)
"""
from __future__ import annotations

import ctypes as C

from . import binding as _b

FLY_CACHE_BF16, FLY_CACHE_E4M3 = 0, 1
FLAG_NOT_WRITTEN = 32

EXPORTS = ("fly_cache_append", "fly_cache_read", "fly_attention_create", "fly_attention_destroy", "fly_attention_run",
           "fly_attention_device_status", "fly_attention_selftest_wait", "fly_attention_last_launch_count", "fly_attention_last_cuda_error")


class fly_cache_t(C.Structure):
    _fields_ = [("device", C.c_int32), ("format", C.c_int),
                ("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p),
                ("num_pages", C.c_int32), ("page_size", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64),
                ("block_table", C.c_void_p), ("table_stride", C.c_int64), ("max_pages", C.c_int32), ("sequences", C.c_int32),
                ("lengths", C.c_void_p)]


class fly_rows_t(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class fly_attention_config_t(C.Structure):
    _fields_ = [("device", C.c_int32), ("max_batch", C.c_int32), ("max_tokens", C.c_int32), ("heads", C.c_int32),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class fly_attention_args_t(C.Structure):
    _fields_ = [("B", C.c_int32), ("n", C.c_int32), ("q", fly_rows_t), ("out", fly_rows_t), ("lse", C.c_void_p),
                ("counts", C.c_void_p), ("window", C.c_int32), ("sinks", C.c_int32), ("scale", C.c_double)]


_lib = None


def lib() -> C.CDLL:
    """libfly_verify.so with the entry points of fly_cache.h declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = _b.lib()
    P = C.POINTER
    L.fly_cache_append.argtypes = [P(fly_cache_t), C.c_int32, C.c_int32, P(fly_rows_t), P(fly_rows_t), C.c_void_p, C.c_void_p, C.c_void_p]
    L.fly_cache_read.argtypes = [P(fly_cache_t), C.c_int32, C.c_int32, C.c_void_p, P(fly_rows_t), P(fly_rows_t), C.c_void_p]
    L.fly_attention_create.argtypes = [P(fly_attention_config_t), P(C.c_void_p)]
    L.fly_attention_destroy.argtypes = [C.c_void_p]
    L.fly_attention_run.argtypes = [C.c_void_p, P(fly_cache_t), P(fly_attention_args_t), C.c_void_p]
    L.fly_attention_device_status.argtypes = [C.c_void_p, C.c_void_p]
    L.fly_attention_selftest_wait.argtypes = [C.c_void_p, C.c_void_p]
    L.fly_attention_last_launch_count.argtypes = [C.c_void_p]
    L.fly_attention_last_cuda_error.argtypes = [C.c_void_p]
    for name in EXPORTS:
        getattr(L, name).restype = C.c_int
    _b._native.init_cache(*[C.cast(getattr(L, f), C.c_void_p).value for f in ("fly_cache_append", "fly_cache_read", "fly_attention_run")])
    _lib = L
    return L


def _expect(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


class _Held(C.Structure):
    """A fly_cache_t that is replaced as a whole by one assignment."""
    _fields_ = [("c", fly_cache_t)]


class PagedCache:
    """A cache over the caller's tensors (kept, not copied):

      k_pages, v_pages    [num_pages, page_size, kv_heads, head_dim], bfloat16 or float8_e4m3fn, alike in their strides; head_dim
                          contiguous, the other dimensions in any order (views of one tensor are fine)
      k_scales, v_scales  [num_pages, kv_heads, page_size] uint8, contiguous; e4m3 only
      block_table         [sequences, max_pages] int32, rows that do not overlap
      lengths             [sequences] int32: positions held, before the chunk of the round

    block_table and lengths can be assigned: calls from then on use the new tensor (a table may be wider than the one before, but is for
    as many sequences).  The others are fixed.  Tensors keep their storage while the cache has them (no resize_, no set_).
    """

    def __init__(self, k_pages, v_pages, block_table, lengths, k_scales=None, v_scales=None):
        import torch
        lib()
        e4m3 = k_pages.dtype == torch.float8_e4m3fn
        _expect(e4m3 or k_pages.dtype == torch.bfloat16, "pages are bfloat16 or float8_e4m3fn")
        _expect(k_pages.dim() == 4 and k_pages.stride(3) == 1, "pages are [num_pages, page_size, kv_heads, head_dim], head_dim contiguous")
        _expect(v_pages.dtype == k_pages.dtype and v_pages.shape == k_pages.shape and v_pages.stride() == k_pages.stride(),
                "k_pages and v_pages are alike in type, shape and strides")
        pages, size, heads, dim = k_pages.shape
        self._check_table(block_table)
        self._check_lengths(lengths, block_table)
        _expect(e4m3 == (k_scales is not None) == (v_scales is not None), "k_scales and v_scales belong to e4m3 pages, and to them only")
        for s in (k_scales, v_scales) if e4m3 else ():
            _expect(s.dtype == torch.uint8 and tuple(s.shape) == (pages, heads, size) and s.is_contiguous(),
                    "scales are [num_pages, kv_heads, page_size] uint8, contiguous")
        tensors = [t for t in (k_pages, v_pages, block_table, lengths, k_scales, v_scales) if t is not None]
        _expect(all(t.is_cuda and t.device == k_pages.device for t in tensors), "all tensors of a cache are on one CUDA device")
        self._pages = k_pages, v_pages, k_scales, v_scales
        self._held = _Held()
        self._at = C.addressof(self._held)
        self._set(block_table, lengths)

    @staticmethod
    def _check_table(t):
        import torch
        _expect(isinstance(t, torch.Tensor) and t.dim() == 2 and t.dtype == torch.int32 and (t.stride(1) == 1 or t.size(1) == 1),
                "block_table is [sequences, max_pages] int32 with contiguous rows")
        _expect(t.size(0) == 1 or t.stride(0) >= t.size(1), "rows of block_table do not overlap (an expanded one: .contiguous())")

    @staticmethod
    def _check_lengths(t, table):
        import torch
        _expect(isinstance(t, torch.Tensor) and t.dtype == torch.int32 and tuple(t.shape) == (table.size(0),) and t.is_contiguous(),
                "lengths is [sequences] int32")

    def _set(self, table, lengths):
        k, v, ks, vs = self._pages
        address = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self._held.c = fly_cache_t(k.device.index, FLY_CACHE_BF16 if ks is None else FLY_CACHE_E4M3, address(k), address(v), address(ks), address(vs),
                                   *k.shape, k.stride(0), k.stride(1), k.stride(2), address(table), max(table.stride(0), table.size(1)),
                                   table.size(1), table.size(0), address(lengths))
        self._block_table, self._lengths = table, lengths

    k_pages = property(lambda self: self._pages[0])
    v_pages = property(lambda self: self._pages[1])
    k_scales = property(lambda self: self._pages[2])
    v_scales = property(lambda self: self._pages[3])
    struct = property(lambda self: self._held.c, doc="The fly_cache_t of the calls.")

    @property
    def block_table(self):
        return self._block_table

    @block_table.setter
    def block_table(self, t):
        self._check_table(t)
        _expect(t.size(0) == self._lengths.size(0), "block_table is for as many sequences as lengths")
        _expect(t.device == self.k_pages.device, "all tensors of a cache are on one CUDA device")
        self._set(t, self._lengths)

    @property
    def lengths(self):
        return self._lengths

    @lengths.setter
    def lengths(self, t):
        self._check_lengths(t, self._block_table)
        _expect(t.device == self.k_pages.device, "all tensors of a cache are on one CUDA device")
        self._set(self._block_table, t)


def cache_append(cache: PagedCache, k, v, counts=None, row_flags=None, stream: int = 0):
    """fly_cache_append: k, v [B, n, kv_heads, head_dim] bf16 (any strides, head_dim contiguous) go to positions lengths[b] + i.
    counts [B] int32: rows that a sequence really has.  row_flags [B, n] int32: FLAG_NOT_WRITTEN where a token found no page."""
    st = _b._native.cache_append(cache._at, k, v, counts, row_flags, stream or 0)
    if st:
        raise _b.FlyError(st, "fly_cache_append")


def cache_read(cache: PagedCache, k_out, v_out, starts=None, stream: int = 0):
    """fly_cache_read: positions starts[b] + i (starts [B] int32, None = 0) into k_out, v_out [B, n, kv_heads, head_dim] bf16; rows of
    positions that a sequence does not hold are left as they are."""
    st = _b._native.cache_read(cache._at, k_out, v_out, starts, stream or 0)
    if st:
        raise _b.FlyError(st, "fly_cache_read")


class ChunkAttention:
    """Handle of one attention shape (fly_attention_create / fly_attention_destroy); its scratch serves one step at a time."""

    def __init__(self, max_batch: int, max_tokens: int, heads: int, kv_heads: int, head_dim: int, device: int = 0):
        self._h = C.c_void_p()
        cfg = fly_attention_config_t(int(device), int(max_batch), int(max_tokens), int(heads), int(kv_heads), int(head_dim))
        st = lib().fly_attention_create(C.byref(cfg), C.byref(self._h))
        if st != _b.FLY_OK:
            self._h = C.c_void_p()
            raise _b.FlyError(st, "fly_attention_create")
        self.heads = int(heads)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().fly_attention_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def last_launch_count(self) -> int:
        return int(lib().fly_attention_last_launch_count(self._h))

    def device_status(self, stream: int = 0) -> int:
        """fly_attention_device_status: synchronises the stream; FLY_OK or FLY_ERR_TIMEOUT."""
        return int(lib().fly_attention_device_status(self._h, C.c_void_p(stream)))

    def selftest_wait(self, stream: int = 0) -> int:
        """fly_attention_selftest_wait: makes one bounded device-side wait run out on purpose (no fault)."""
        return int(lib().fly_attention_selftest_wait(self._h, C.c_void_p(stream)))

    def run(self, cache: PagedCache, q, out, window: int = 0, sinks: int = 0, scale: float = 0.0, counts=None, lse=None, stream: int = 0):
        """fly_attention_run: q [B, n, heads, head_dim] bf16 -> out, alike; the chunk has been appended behind cache.lengths.
        window: 0, or how many positions up to its own a row sees; sinks: first positions that stay visible with a window.
        scale: 0 = 1 / sqrt(head_dim).  counts [B] int32 as in cache_append.  lse [B, n, heads] fp32: logarithm of the softmax's sum."""
        st = _b._native.attention_run(self._h.value or 0, cache._at, self.heads, q, out, window, sinks, scale, counts, lse, stream or 0)
        if st:
            raise _b.FlyError(st, "fly_attention_run", lib().fly_attention_last_cuda_error(self._h))
        return out
