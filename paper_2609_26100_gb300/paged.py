"""The paged 4-bit KV cache for PyTorch users: tensors and streams are torch's, all work runs in
libtss.so (tss_paged_*, tss_pages_*).

``PagePool`` keeps the books of pages of any content (page table, pages held, reference counts, all on the
device); ``Kv4Cache`` appends to, reads and attends over pages held in 4 bits.  Both work on the caller's
tensors; ``Kv4Cache.allocate`` makes a set that fits together.  All tensors are on the pool's GPU, which has to
be the current device in every call.
"""
from __future__ import annotations

import ctypes
from array import array
from typing import Optional, Sequence

import torch

from . import native
from .native import _P, _ptr, check, lib

PAGE_TOKENS = native.PAGE_TOKENS
_CODES = {torch.bfloat16: native.TSS_DTYPE_BF16, torch.float16: native.TSS_DTYPE_F16, torch.float32: native.TSS_DTYPE_F32}


def page_bytes(n_kv_heads: int, head_dim: int) -> int:
    """Bytes of one 4-bit page (64 tokens of every KV head of one layer)."""
    n = lib().tss_paged_page_bytes(n_kv_heads, head_dim)
    if n == 0:
        raise ValueError(f"no 4-bit page for {n_kv_heads} heads of {head_dim}")
    return n


def pages_for(tokens: int) -> int:
    return -(-int(tokens) // PAGE_TOKENS)


def _pages(tokens) -> list:
    """Pages of each length; -1, which the library refuses, for one below zero (rounding up would make some of them 0)."""
    return [-(-t // PAGE_TOKENS) if t >= 0 else -1 for t in tokens]


def _row_stride(t: torch.Tensor, shape, device: int, what: str) -> int:
    """Elements between the rows of t, a tensor on that GPU which has the given shape and contiguous heads."""
    if t.shape != shape or t.get_device() != device:
        raise ValueError(f"{what}: {list(shape)} on the pool's GPU is wanted")
    row, head, one = t.stride()
    n, h, d = shape
    if n == 0:
        return h * d
    if one != 1 or (h > 1 and head != d):
        raise ValueError(f"{what}: the heads of a row must be contiguous")
    return row if n > 1 else h * d  # (nothing steps from a single row)


def _code(t: torch.Tensor) -> int:
    try:
        return _CODES[t.dtype]
    except KeyError:
        raise TypeError(f"bfloat16, float16 or float32 is wanted, not {t.dtype}") from None


def _host(values) -> array:
    """int32 values for a call that reads them before it returns (pass its address, keep it until then)."""
    return array("i", values)


def _ints(t: torch.Tensor, shape, device: int, what: str) -> None:
    if t.shape != shape or t.dtype != torch.int32 or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{what}: contiguous int32 {list(shape)} on the pool's GPU is wanted")


def _stream_of(device: int, stream) -> int:
    """The stream of a call on that device (None: torch's current one), which has to be the current device."""
    if torch.cuda.current_device() != device:
        raise ValueError(f"the pool is on cuda:{device}, which is not the current device")
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream


def _layers(pool: torch.Tensor):
    """(array of each layer's address, layers, pages, bytes of a page) of a tensor [layers][pages][...]."""
    if pool.dim() < 3 or not pool.is_contiguous() or not pool.is_cuda:
        raise ValueError("pool: contiguous [layers][pages][...] on the GPU is wanted")
    n, step = pool.shape[0], pool.stride(0) * pool.element_size()
    ptrs = (_P * n)(*[pool.data_ptr() + i * step for i in range(n)])
    return ptrs, n, pool.shape[1], pool.stride(1) * pool.element_size()


class PagePool:
    """Page table [seqs][max_pages], pages held [seqs] and reference counts [pages] (int32, on the GPU) of a
    pool [layers][pages][...].  Calls are enqueued on torch's current stream (or `stream`); a failure that
    only the device sees is reported by sync_status()."""

    def __init__(self, pool: torch.Tensor, table: torch.Tensor, held: torch.Tensor, refs: torch.Tensor):
        self._ptrs, self.n_layers, self.n_pages, self.page_bytes = _layers(pool)
        if table.dim() != 2:
            raise ValueError("table: int32 [seqs][max_pages] is wanted")
        self.n_seqs, self.max_pages = table.shape
        self._dev = dev = pool.get_device()
        _ints(table, (self.n_seqs, self.max_pages), dev, "table")
        _ints(held, (self.n_seqs,), dev, "held")
        _ints(refs, (self.n_pages,), dev, "refs")
        self.pool, self.table, self.held, self.refs = pool, table, held, refs
        self._tables = native.TssPageTables(table.data_ptr(), held.data_ptr(), refs.data_ptr())
        self._ref = ctypes.byref(self._tables)
        h = _P()
        self._c_free, self._c_fork = lib().tss_pages_free, lib().tss_pages_fork
        with torch.cuda.device(dev):
            check(lib().tss_pages_create(self.n_seqs, self.max_pages, self.n_pages, ctypes.byref(h)), "tss_pages_create")
        self._h = h

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().tss_pages_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self, stream):
        return _stream_of(self._dev, stream)

    def reserve(self, seqs: Sequence[int], tokens: Sequence[int], stream=None) -> None:
        """Pages for tokens[i] tokens of seqs[i] (those it holds stay)."""
        if len(seqs) != len(tokens):
            raise ValueError("seqs and tokens differ in length")
        a, b = _host(seqs), _host(_pages(tokens))
        check(lib().tss_pages_reserve(self._h, self._ref, len(a), a.buffer_info()[0], b.buffer_info()[0], self._stream(stream)),
              "tss_pages_reserve")

    def free(self, seqs: Sequence[int], tokens: Optional[Sequence[int]] = None, stream=None) -> None:
        """Give back the pages of seqs[i] past its first tokens[i] tokens (None: all)."""
        if tokens is not None and len(seqs) != len(tokens):
            raise ValueError("seqs and tokens differ in length")
        a, keep = _host(seqs), None
        if tokens is not None:
            keep = _host(_pages(tokens))
        s = self._c_free(self._h, self._ref, len(a), a.buffer_info()[0], None if keep is None else keep.buffer_info()[0],
                         self._stream(stream))
        if s:
            check(s, "tss_pages_free")

    def fork(self, src: Sequence[int], dst: Sequence[int], tokens: Sequence[int], stream=None) -> None:
        """dst[i] (which holds nothing) becomes the first tokens[i] tokens of src[i]: full pages are shared, a
        part-filled last one is copied."""
        n = len(src)
        if len(dst) != n or len(tokens) != n:
            raise ValueError("src, dst and tokens differ in length")
        # src, dst, pages to share and pages in all, in one array
        a = _host((*src, *dst, *[t // PAGE_TOKENS for t in tokens], *_pages(tokens)))
        at, step = a.buffer_info()[0], n * a.itemsize
        s = self._c_fork(self._h, self._ref, self._ptrs, self.n_layers, self.page_bytes, n, at, at + step, at + 2 * step, at + 3 * step,
                         self._stream(stream))
        if s:
            check(s, "tss_pages_fork")

    def compact(self, table_out: Optional[torch.Tensor] = None, refs_out: Optional[torch.Tensor] = None, stream=None) -> None:
        """Move the pages in use to the lowest ids; the new table and counts replace the pool's, or go to the
        given tensors."""
        t, r = (self.table if table_out is None else table_out), (self.refs if refs_out is None else refs_out)
        _ints(t, self.table.shape, self._dev, "table_out")
        _ints(r, self.refs.shape, self._dev, "refs_out")
        check(lib().tss_pages_compact(self._h, self._ref, t.data_ptr(), r.data_ptr(), self._ptrs, self.n_layers,
                                      self.page_bytes, self._stream(stream)), "tss_pages_compact")

    def copy(self, src: torch.Tensor, dst: torch.Tensor, stream=None) -> None:
        """Copy page src[i] over page dst[i] in every layer (int32 tensors on the GPU)."""
        _ints(src, (src.numel(),), self._dev, "src")
        _ints(dst, (src.numel(),), self._dev, "dst")
        check(lib().tss_pages_copy(self._h, self._ptrs, self.n_layers, self.page_bytes, src.numel(), _ptr(src), _ptr(dst),
                                   self._stream(stream)), "tss_pages_copy")

    def sync_status(self, stream=None) -> int:
        return lib().tss_pages_sync_status(self._h, self._stream(stream))


class Kv4Cache:
    """A KV cache in 4 bits: pool uint8 [layers][pages][page bytes], table int32 [seqs][max_pages]."""

    def __init__(self, pool: torch.Tensor, table: torch.Tensor, *, n_q_heads: int, n_kv_heads: int, head_dim: int):
        if pool.dtype != torch.uint8 or pool.dim() != 3 or pool.shape[2] != page_bytes(n_kv_heads, head_dim):
            raise ValueError("pool: uint8 [layers][pages][page bytes] is wanted")
        if table.dim() != 2:
            raise ValueError("table: int32 [seqs][max_pages] is wanted")
        self._dev = pool.get_device()
        _ints(table, table.shape, self._dev, "table")
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim
        self.pool, self.table = pool, table
        self._ptrs, n_layers, n_pages, _ = _layers(pool)
        self._cache = native.TssPagedCache(ctypes.cast(self._ptrs, ctypes.POINTER(_P)), n_layers, n_pages, table.data_ptr(),
                                           table.shape[0], table.shape[1])
        self._cache_ref = ctypes.byref(self._cache)
        self._c_append, self._c_read, self._c_attention = lib().tss_paged_append, lib().tss_paged_read, lib().tss_paged_attention
        self.pages: Optional[PagePool] = None
        h = _P()
        with torch.cuda.device(self._dev):
            check(lib().tss_paged_create(n_q_heads, n_kv_heads, head_dim, ctypes.byref(h)), "tss_paged_create")
        self._h = h

    @classmethod
    def allocate(cls, *, n_layers: int, n_pages: int, n_seqs: int, max_pages: int, n_q_heads: int, n_kv_heads: int,
                 head_dim: int, device: str = "cuda") -> "Kv4Cache":
        """An empty cache with its page books (the result's `pages`)."""
        pool = torch.zeros((n_layers, n_pages, page_bytes(n_kv_heads, head_dim)), dtype=torch.uint8, device=device)
        table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device)
        c = cls(pool, table, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim)
        c.pages = PagePool(pool, table, torch.zeros(n_seqs, dtype=torch.int32, device=device),
                           torch.zeros(n_pages, dtype=torch.int32, device=device))
        return c

    def close(self) -> None:
        if self.pages is not None:
            self.pages.close()
        if getattr(self, "_h", None):
            lib().tss_paged_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @staticmethod
    def batch(seqs: Sequence[int], first: Sequence[int], n_tokens: Sequence[int]) -> native.TssPagedBatch:
        """Request i is the tokens [first[i], first[i] + n_tokens[i]) of sequence seqs[i]."""
        if not len(seqs) == len(first) == len(n_tokens):
            raise ValueError("seqs, first and n_tokens differ in length")
        keep = [_host(map(int, x)) for x in (seqs, first, n_tokens)]  # (OverflowError past 32 bits)
        b = native.TssPagedBatch(len(seqs), *[a.buffer_info()[0] for a in keep])
        b._keep = keep
        b.ref = ctypes.byref(b)
        b.rows = sum(int(n) for n in n_tokens)
        return b

    def append(self, layer: int, batch, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """Quantise k, v [rows][kv heads][head_dim] into the pages of the batch's tokens."""
        shape, dev = (batch.rows, self.n_kv_heads, self.head_dim), self._dev
        if k.dtype != v.dtype:
            raise ValueError("k and v differ in type")
        s = self._c_append(self._h, self._cache_ref, layer, batch.ref, k.data_ptr(), v.data_ptr(), _row_stride(k, shape, dev, "k"),
                           _row_stride(v, shape, dev, "v"), _code(k), _stream_of(self._dev, stream))
        if s:
            check(s, "tss_paged_append")

    def read(self, layer: int, batch, k: Optional[torch.Tensor], v: Optional[torch.Tensor], stream=None) -> None:
        """The values that the batch's tokens are held as, to k and v (either may be None)."""
        shape, dev = (batch.rows, self.n_kv_heads, self.head_dim), self._dev
        one = k if k is not None else v
        if one is None or (k is not None and v is not None and k.dtype != v.dtype):
            raise ValueError("k or v is wanted, of one type")
        s = self._c_read(self._h, self._cache_ref, layer, batch.ref, None if k is None else k.data_ptr(),
                         None if v is None else v.data_ptr(), 0 if k is None else _row_stride(k, shape, dev, "k"),
                         0 if v is None else _row_stride(v, shape, dev, "v"), _code(one), _stream_of(self._dev, stream))
        if s:
            check(s, "tss_paged_read")

    def attention(self, layer: int, batch, q: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor] = None, *,
                  scale: Optional[float] = None, window: int = 0, sinks: int = 0, mask: Optional[torch.Tensor] = None,
                  positions: Optional[torch.Tensor] = None, stream=None) -> None:
        """Attention of the batch's rows (already appended) over their sequences: q, out [rows][heads][head_dim];
        lse float32 [rows][heads]; mask int64 [rows][2] (bits of the block's rows that a row sees; None: a chain);
        window and sinks as in tss_paged_attention, positions int32 [rows]."""
        n, h, d = shape = (batch.rows, self.n_q_heads, self.head_dim)
        dev = self._dev
        if out.dtype != q.dtype:
            raise ValueError("out: the type of q is wanted")
        if lse is not None and (lse.shape != (n, h) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.get_device() != dev):
            raise ValueError("lse: contiguous float32 [rows][heads] on the pool's GPU is wanted")
        if mask is not None and (mask.shape != (n, 2) or mask.dtype not in (torch.int64, torch.uint64) or not mask.is_contiguous()
                                 or mask.get_device() != dev):
            raise ValueError("mask: contiguous 64-bit [rows][2] on the pool's GPU is wanted")
        if positions is not None:
            _ints(positions, (n,), dev, "positions")
        a = native.TssPagedAttn(q.data_ptr(), _row_stride(q, shape, dev, "q"), out.data_ptr(), _row_stride(out, shape, dev, "out"),
                                None if lse is None else lse.data_ptr(), _code(q), d ** -0.5 if scale is None else scale, window,
                                sinks, None if mask is None else mask.data_ptr(), None if positions is None else positions.data_ptr())
        s = self._c_attention(self._h, self._cache_ref, layer, batch.ref, ctypes.byref(a),
                              _stream_of(self._dev, stream))
        if s:
            check(s, "tss_paged_attention")

    def inject_timeout(self, n_calls: int) -> None:
        """tss_paged_inject_timeout: make a wait of the next n_calls attention calls run out (tests)."""
        check(lib().tss_paged_inject_timeout(self._h, n_calls), "tss_paged_inject_timeout")

    def sync_status(self, stream=None) -> int:
        return lib().tss_paged_sync_status(self._h, _stream_of(self._dev, stream))
