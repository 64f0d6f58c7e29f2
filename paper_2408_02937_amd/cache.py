"""Binding of include/rtams_cache.h: a paged cache of attention keys and values held in 4 bits, and the attention that
reads it, beside the index of rtams.py.

Like the index, argument marshalling only: every step runs in the HIP kernels behind the C ABI, calls are asynchronous on
the stream given (the current one unless told), there is no fallback.  Tensors handed to a call on a stream given are kept for that
stream: they may be dropped when the call has returned.  Nothing here has a gradient, and a tensor that asks for one is refused.

    c = Cache(kv_heads=8, head_dim=128, layers=2, pages=4096, max_seqs=64)
    c.extend(seqs, starts)                              # room for the new rows of these sequences
    for layer in range(2):
        c.write(layer, k, v, seqs, starts, max_new)     # k, v [rows][8][128] bfloat16 or float16
        out = c.attend(layer, q, seqs, starts, max_new) # q [rows][heads][128], a multiple of 8 heads
    c.fork(src, dst)                                    # branches share pages until they grow
    c.trim(seqs)                                        # ... and are freed
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional, Tuple

import torch

from paper_2408_02937_amd import rtams
from paper_2408_02937_amd.rtams import CacheConfig, CacheQuery, CacheView, _chk, _device_bytes, lib

_query = struct.Struct("@iiiiiifPqqPqqP").pack  # CacheQuery, three times as fast as its fields one by one
assert struct.calcsize("@iiiiiifPqqPqqP") == C.sizeof(CacheQuery)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


class Cache:
    """rtams_cache over a pool and a scratch tensor that this object keeps alive."""

    def __init__(self, kv_heads: int, head_dim: int, layers: int = 1, page_tokens: int = 64, pages: Optional[int] = None,
                 pool_bytes: Optional[int] = None, max_seqs: int = 256, max_pages: Optional[int] = None, device: str = "cuda:0"):
        """pages: of page_tokens tokens of all layers, shared by all sequences (or pool_bytes, tables included); max_pages: of one
        sequence (default: all)."""
        L = lib()
        self.kv_heads, self.head_dim, self.layers, self.page_tokens, self.max_seqs = kv_heads, head_dim, layers, page_tokens, max_seqs
        self.device = torch.device(device)
        self.device = torch.device(self.device.type, torch.cuda.current_device() if self.device.index is None else self.device.index)
        if pages is None and pool_bytes is None:
            raise ValueError("give pages or pool_bytes")
        if max_pages is None:
            if pages is None:
                raise ValueError("give max_pages with pool_bytes")
            max_pages = pages
        cfg = CacheConfig(layers=layers, kv_heads=kv_heads, head_dim=head_dim, page_tokens=page_tokens, max_seqs=max_seqs, max_pages=max_pages)
        if pool_bytes is None:
            pool_bytes = L.rtams_cache_pool_bytes_for(C.byref(cfg), pages)
        scratch_bytes = L.rtams_cache_scratch_bytes_for(C.byref(cfg))
        if pool_bytes == 0 or scratch_bytes == 0:
            raise rtams.RtamsError(rtams.EINVAL, "cache_pool_bytes_for", L.rtams_last_error().decode())
        self.pool = _device_bytes(pool_bytes, self.device)
        self.scratch = _device_bytes(scratch_bytes, self.device)
        cfg.d_pool, cfg.pool_bytes = self.pool.data_ptr(), pool_bytes
        cfg.d_scratch, cfg.scratch_bytes = self.scratch.data_ptr(), scratch_bytes
        h = C.c_void_p()
        torch.cuda.synchronize(self.device)
        _chk(L.rtams_cache_create(C.byref(cfg), C.byref(h)), "rtams_cache_create")
        self._h, self._lib = h, L
        v = CacheView()
        _chk(L.rtams_cache_layout(h, C.byref(v)), "rtams_cache_layout")
        base = self.pool.data_ptr()

        def words(at, *shape):
            n = 1
            for x in shape:
                n *= x
            return self.pool[at - base:at - base + 4 * n].view(torch.int32).view(*shape)

        # views of the pool, for reading; what a call on a stream left is there for work behind it on that stream
        self.table = words(v.d_table, max_seqs, max_pages)   # page numbers, -1 behind a sequence's last
        self.lengths = words(v.d_lengths, max_seqs)          # tokens
        self.refs = words(v.d_refs, v.pages)                 # table entries that name a page
        at = v.d_pages - base
        self.pages = self.pool[at:at + layers * v.pages * v.page_bytes].view(layers, v.pages, v.page_bytes)

    def close(self):
        if getattr(self, "_h", None):
            lib().rtams_cache_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- arguments
    def _stream(self, stream) -> int:
        return _current_stream(self.device.index) if stream is None else stream.cuda_stream

    def _ints(self, t: Optional[torch.Tensor], what: str, n: Optional[int] = None, stream=None) -> Optional[int]:
        if t is None:
            return None
        if not (t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous() and t.device == self.device and (n is None or t.shape[0] == n)):
            raise ValueError(f"{what} must be a contiguous int32 tensor on {self.device}" + ("" if n is None else f" of {n} entries"))
        if stream is not None:
            t.record_stream(stream)
        return t.data_ptr()

    def _items(self, seqs, starts, n, max_new, stream):
        """(n, pointers of seqs and starts, most rows of an item)."""
        if n is None:
            n = seqs.shape[0] if seqs is not None else starts.shape[0] - 1 if starts is not None else None
        if n is None or n < 0:
            raise ValueError("give seqs, starts or n")
        if starts is None:
            max_new = 1
        elif max_new is None:
            raise ValueError("with starts, give max_new: the most rows of one item")
        return n, self._ints(seqs, "seqs", n, stream), self._ints(starts, "starts", n + 1, stream), max_new

    def _rows(self, t: torch.Tensor, heads: Optional[int], what: str, stream=None) -> torch.Tensor:
        if not (t.dim() == 3 and t.shape[2] == self.head_dim and (heads is None or t.shape[1] == heads) and t.dtype in (torch.bfloat16, torch.float16)
                and t.device == self.device and (t.stride(2) == 1 or t.numel() == 0)):
            raise ValueError(f"{what} must be a bfloat16 or float16 tensor [rows][{'heads' if heads is None else heads}][{self.head_dim}] on {self.device} "
                             "whose channels lie next to each other")
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{what} asks for a gradient, which no call on the cache has: detach it, or call under torch.no_grad()")
        if stream is not None:
            t.record_stream(stream)
        return t

    def _alike(self, k: torch.Tensor, v: torch.Tensor, stream):
        places = lambda t: [t.stride(d) for d in (0, 1) if t.shape[d] > 1]
        if k.numel() == 0 or (places(k) == places(v) and (k.shape[0] == 1 or k.stride(0) < 1 << 24)):
            return k, v
        if stream is None:
            return k.contiguous(), v.contiguous()
        with torch.cuda.stream(stream):
            return k.contiguous(), v.contiguous()

    def _empty(self, shape, dtype: torch.dtype, stream) -> torch.Tensor:
        """Memory for an output on a stream given: that stream's own, since what is free on the current one may still be read there by work under
        way, and not used again before the current stream, where the caller has it, is done with it."""
        with torch.cuda.stream(stream):
            t = torch.empty(shape, dtype=dtype, device=self.device)
        t.record_stream(torch.cuda.current_stream(self.device))
        return t

    # ---- the path
    def extend(self, seqs: Optional[torch.Tensor] = None, starts: Optional[torch.Tensor] = None, n: Optional[int] = None, stream=None) -> None:
        """Room for the items' rows (one each without starts) at the ends of their sequences."""
        n, sp, tp, _ = self._items(seqs, starts, n, 1, stream)
        _chk(self._lib.rtams_cache_extend(self._h, n, sp, tp, self._stream(stream)), "rtams_cache_extend")

    def write(self, layer: int, k: torch.Tensor, v: torch.Tensor, seqs: Optional[torch.Tensor] = None, starts: Optional[torch.Tensor] = None,
              max_new: Optional[int] = None, stream=None) -> None:
        """Keys and values of the sequences' last rows, [rows][kv_heads][head_dim].  The kernel takes both at the same strides, rows less than 2^24
        elements apart; where they are not (keys that were turned, values still in a projection's output), copies are made first."""
        k, v = self._rows(k, self.kv_heads, "k", stream), self._rows(v, self.kv_heads, "v", stream)
        if k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v must have the same shape and type")
        rows = k.shape[0]
        strides = k.stride()
        if strides != v.stride() or strides[0] >= 1 << 24:
            k, v = self._alike(k, v, stream)
            strides = k.stride()
        n, sp, tp, max_new = self._items(seqs, starts, rows if seqs is None and starts is None else None, max_new, stream)
        _chk(self._lib.rtams_cache_write(self._h, layer, n, sp, tp, rows, max_new, k.data_ptr(), v.data_ptr(), strides[0], strides[1],
                                     _TYPES[k.dtype], self._stream(stream)), "rtams_cache_write")

    def read(self, layer: int, rows: int, seqs: Optional[torch.Tensor] = None, starts: Optional[torch.Tensor] = None,
             max_new: Optional[int] = None, dtype: torch.dtype = torch.float32, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """What the cache holds of the sequences' last rows, as values."""
        if dtype not in _TYPES:
            raise ValueError("dtype must be bfloat16, float16 or float32")
        n, sp, tp, max_new = self._items(seqs, starts, rows if seqs is None and starts is None else None, max_new, stream)
        shape = (rows, self.kv_heads, self.head_dim)
        if stream is None:
            k = torch.empty(shape, dtype=dtype, device=self.device)
            v = torch.empty_like(k)
        else:
            k, v = self._empty(shape, dtype, stream), self._empty(shape, dtype, stream)
        _chk(self._lib.rtams_cache_read(self._h, layer, n, sp, tp, rows, max_new, k.data_ptr(), v.data_ptr(), _TYPES[dtype], self._stream(stream)),
             "rtams_cache_read")
        return k, v

    def attend(self, layer: int, q: torch.Tensor, seqs: Optional[torch.Tensor] = None, starts: Optional[torch.Tensor] = None,
               max_new: Optional[int] = None, scale: Optional[float] = None, causal: bool = True, window: int = 0,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of the sequences' last rows, q [rows][heads][head_dim]; lse: float32 [rows][heads] that takes the
        logarithms of the sums of exp(score)."""
        q = self._rows(q, None, "q", stream)
        rows, heads = q.shape[0], q.shape[1]
        n, sp, tp, max_new = self._items(seqs, starts, rows if seqs is None and starts is None else None, max_new, stream)
        if out is None:
            shape = (rows, heads, self.head_dim)
            out = q.new_empty(shape) if stream is None else self._empty(shape, q.dtype, stream)
        elif self._rows(out, heads, "out", stream).shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out must have the shape and type of q")
        lp = None
        if lse is not None:
            if not (lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (rows, heads) and lse.device == self.device):
                raise ValueError("lse must be a contiguous float32 tensor [rows][heads]")
            if stream is not None:
                lse.record_stream(stream)
            lp = lse.data_ptr()
        cq = _query(layer, heads, _TYPES[q.dtype], int(causal), window, max_new, self.head_dim ** -0.5 if scale is None else scale,
                        q.data_ptr(), q.stride(0), q.stride(1), out.data_ptr(), out.stride(0), out.stride(1), lp or 0)
        _chk(self._lib.rtams_cache_attend(self._h, cq, n, sp, tp, rows, self._stream(stream)), "rtams_cache_attend")
        return out

    # ---- pages
    def fork(self, src: torch.Tensor, dst: torch.Tensor, copy: bool = False, stream=None) -> None:
        """Empty sequences dst become what src are, sharing pages until they grow, or (copy) in pages of their own."""
        n = src.shape[0]
        _chk(self._lib.rtams_cache_fork(self._h, n, self._ints(src, "src", None, stream), self._ints(dst, "dst", n, stream), int(copy), self._stream(stream)), "rtams_cache_fork")

    def trim(self, seqs: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None, n: Optional[int] = None, stream=None) -> None:
        """Cuts sequences down to `lengths` tokens (without: to none)."""
        if n is None:
            n = seqs.shape[0] if seqs is not None else lengths.shape[0] if lengths is not None else None
        if n is None:
            raise ValueError("give seqs, lengths or n")
        _chk(self._lib.rtams_cache_trim(self._h, n, self._ints(seqs, "seqs", n, stream), self._ints(lengths, "lengths", n, stream), self._stream(stream)), "rtams_cache_trim")

    def compact(self, stream=None) -> None:
        """Moves the pages in use to the front of the pool."""
        _chk(self._lib.rtams_cache_compact(self._h, self._stream(stream)), "rtams_cache_compact")

    # ---- introspection
    @property
    def free_pages(self) -> int:
        v = C.c_int64()
        _chk(self._lib.rtams_cache_free_pages(self._h, C.byref(v)), "rtams_cache_free_pages")
        return v.value

    def poll_error(self) -> int:
        return self._lib.rtams_cache_poll_error(self._h)

    def clear_error(self) -> None:
        _chk(self._lib.rtams_cache_clear_error(self._h), "rtams_cache_clear_error")
