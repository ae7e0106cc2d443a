"""The paged KV cache around the verify step (speccache.h): page pools, the
operators on them, and the page bookkeeping.  Argument marshalling only; the
operators run in the library's HIP kernels, the bookkeeping in its C++.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B
from .batch import StagingRing

_DTYPE = {torch.bfloat16: B.SPEC_BF16, torch.float32: B.SPEC_F32}
_HERE = contextlib.nullcontext()
_kept = []                             # what objects that ended inside a graph capture held, until the next object


def _stride(t: torch.Tensor, dim: int, otherwise: int) -> int:
    """A dimension's stride; of a dimension that holds one entry (or none) any
    will do, and torch may have any."""
    return t.stride(dim) if t.shape[dim] > 1 else otherwise


def _alike(a: torch.Tensor, b: torch.Tensor) -> bool:
    """The same shape, and the same strides where these matter."""
    return a.shape == b.shape and (a.stride() == b.stride() or all(
        x == y for n, x, y in zip(a.shape, a.stride(), b.stride()) if n > 1))


def _current_raw_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


# torch's own short way to the handle, where it has it (2 us less a call)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_raw_stream)


def _let_go() -> None:
    """What ended objects held goes back once their last calls have ended; not
    in a capture, where nothing may be waited for."""
    if _kept and not torch.cuda.is_current_stream_capturing():
        for _ in range(len(_kept)):
            try:
                held = _kept.pop()         # other threads' objects end here too
            except IndexError:
                return
            held[0].synchronize()


class Pages:
    """Which sequence holds which page (spec_pages_*)."""

    def __init__(self, num_pages: int, page_tokens: int):
        self._h = C.c_void_p()
        self._lib = B.load()
        B.check(self._lib.spec_pages_create(B.int32(num_pages), B.int32(page_tokens), C.byref(self._h)),
                "spec_pages_create")
        self.num_pages, self.page_tokens = num_pages, page_tokens

    def __del__(self):
        if getattr(self, "_h", None):
            self._lib.spec_pages_destroy(self._h)
            self._h = None

    def open(self) -> int:
        s = C.c_int32()
        B.check(self._lib.spec_pages_open(self._h, C.byref(s)), "spec_pages_open")
        return s.value

    def resize(self, sequence: int, tokens: int):
        """The sequence has `tokens` rows from now on.  Returns the page copy
        (src, dst, tokens) to make before rows are written, or None."""
        c = B.SpecPageCopy()
        B.check(self._lib.spec_pages_resize(self._h, B.int32(sequence), B.int32(tokens), C.byref(c)),
                "spec_pages_resize")
        return (c.src, c.dst, c.tokens) if c.tokens else None

    def fork(self, sequence: int) -> int:
        s = C.c_int32()
        B.check(self._lib.spec_pages_fork(self._h, B.int32(sequence), C.byref(s)), "spec_pages_fork")
        return s.value

    def close(self, sequence: int) -> None:
        B.check(self._lib.spec_pages_close(self._h, B.int32(sequence)), "spec_pages_close")

    def table(self, sequence: int) -> np.ndarray:
        n, s = C.c_int32(), B.int32(sequence)
        st = self._lib.spec_pages_table(self._h, s, None, 0, C.byref(n))     # their number
        out = np.empty(n.value, np.int32)
        if st == B.SPEC_ERR_WORKSPACE:
            st = self._lib.spec_pages_table(self._h, s, out.ctypes.data, out.size, C.byref(n))
        B.check(st, "spec_pages_table")
        return out

    def block_table(self, sequences: Sequence[int], block_stride: Optional[int] = None) -> np.ndarray:
        """The sequences' page ids [len(sequences), block_stride], zeros behind them."""
        rows = [self.table(s) for s in sequences]
        longest = max([r.size for r in rows] + [1])
        width = block_stride or longest
        if width < longest:
            raise ValueError("a sequence has more pages than the table has columns")
        out = np.zeros((len(rows), width), np.int32)
        for i, r in enumerate(rows):
            out[i, :r.size] = r
        return out

    def compact(self) -> np.ndarray:
        """Moves used pages to the front of the pool: the copies [n, 3] to make."""
        n = C.c_int32()
        out = np.empty((self.num_pages // 2 + 1, 3), np.int32)
        B.check(self._lib.spec_pages_compact(self._h, out.ctypes.data, out.shape[0], C.byref(n)),
                "spec_pages_compact")
        return out[:n.value].copy()

    @property
    def free(self) -> int:
        return int(self._lib.spec_pages_free_count(self._h))


class PagedCache:
    """Page pools k, v [layers, num_pages, page_tokens, Hkv, d] (bf16 or fp32,
    last dimension contiguous, a page's rows apart by one stride), and the
    block table int32 [requests, pages of the longest] on the same device, its
    rows apart by any stride (it may be replaced: `table`).  An object is used
    by one thread at a time.

    A call runs on `stream`, or the current one, after what is on it already.
    Pools and table are recorded on that stream, so that their memory is not
    given away under a call; the other tensors of a call (new rows, queries,
    outputs, accepted nodes) are its caller's to order and to keep, as for any
    work on a stream that is not their own."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: Optional[torch.Tensor] = None):
        if k.dim() != 5 or k.dtype != v.dtype or k.device != v.device or not _alike(k, v):
            raise ValueError("k and v are [layers, num_pages, page_tokens, Hkv, d] of the same type, strides and device")
        if k.dtype not in _DTYPE:
            raise ValueError("bf16 or fp32 pools")
        if _stride(k, 4, 1) != 1 or (k.shape[1] > 1 and k.stride(1) != k.shape[2] * k.stride(2)):
            raise ValueError("rows are contiguous and pages follow each other")
        self.k, self.v, self.device, self.dtype = k, v, k.device, k.dtype
        self._index = k.device.index
        self._head = k.shape[3:]
        self._width = k.shape[3] * k.shape[4]
        self._lib = B.load()
        c = self.c = B.SpecCache()
        self._ref = C.byref(c)
        self._append = B.SpecAppendArgs()
        self._append_ref = C.byref(self._append)
        c.num_layers, c.num_pages, c.page_tokens, c.num_kv_heads, c.head_dim = k.shape
        c.dtype = _DTYPE[k.dtype]
        c.k, c.v = k.data_ptr(), v.data_ptr()
        c.layer_stride, c.kv_stride_tok = k.stride(0), k.stride(2)
        c.kv_stride_head = _stride(k, 3, c.head_dim)
        self.table = table

    @property
    def table(self) -> Optional[torch.Tensor]:
        return self._table

    @table.setter
    def table(self, t: Optional[torch.Tensor]) -> None:
        if t is not None:
            if t.dim() != 2 or t.dtype != torch.int32 or t.device != self.device or _stride(t, 1, 1) != 1:
                raise ValueError("the block table is int32 [requests, pages] on the pools' device")
            if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
                raise ValueError("the block table's rows overlap")
        # one row's stride is its width (a table of one row may have any)
        width = 0 if t is None else B.int32(t.shape[1])
        stride = B.int32(t.stride(0)) if width and t.shape[0] > 1 else width
        self._table = t
        self._streams = {}                 # the streams that table and pools are recorded on, by their handles
        self._rows = 0 if t is None else t.shape[0]
        self.c.block_table = t.data_ptr() if t is not None else None
        self.c.block_width = width
        self.c.block_stride = stride

    def _enter(self):
        """The pools' device made current for a call (a context)."""
        if self._index is None:
            raise ValueError("the pools are not in device memory")
        return _HERE if torch.cuda.current_device() == self._index else torch.cuda.device(self._index)

    def _stream(self, stream) -> int:
        h = _current_raw_stream(self._index) if stream is None else stream.cuda_stream
        if h not in self._streams:
            self._record(h, stream or torch.cuda.current_stream(self._index))
        return h

    def _record(self, h: int, stream: torch.cuda.Stream) -> None:
        for t in (self.k, self.v, self._table):
            if t is not None:
                t.record_stream(stream)
        self._streams[h] = stream

    def _requests(self, n: int) -> None:
        if self._table is None or n > self._rows:
            raise ValueError("the block table has no row for every request")

    def append(self, chunks: B.SpecChunks, k_new: torch.Tensor, v_new: torch.Tensor, layer: int = 0,
               stream: Optional[torch.cuda.Stream] = None) -> None:
        """Rows k_new, v_new [layers, rows, Hkv, d] (or [rows, Hkv, d]: one layer)
        to the ends of the requests, in the cache's layers from `layer` on."""
        shape, st = k_new.shape, k_new.stride()
        if not _alike(k_new, v_new) or len(shape) not in (3, 4) or \
                shape[-2:] != self._head or shape[-3] < chunks.rows or (st[-1] != 1 and shape[-1] > 1):
            raise ValueError("k_new and v_new are [layers, rows, Hkv, d], a row for every new token")
        if k_new.dtype != self.dtype or v_new.dtype != self.dtype or k_new.device != self.device or \
                v_new.device != self.device:
            raise ValueError("k_new and v_new have the pools' type and device")
        self._requests(chunks.num_requests)
        a = self._append
        a.layer, a.num_layers = B.int32(layer), shape[0] if len(shape) == 4 else 1
        a.k_new, a.v_new = k_new.data_ptr(), v_new.data_ptr()
        width = self._width
        a.new_stride_layer = st[0]
        a.new_stride_tok = st[-3] if shape[-3] > 1 else width
        a.new_stride_head = st[-2] if shape[-2] > 1 else shape[-1]
        with self._enter():
            B.check(self._lib.spec_cache_append(chunks, self._ref, self._append_ref, self._stream(stream)),
                    "spec_cache_append")

    def commit(self, req: B.SpecRequests, accepted_node: torch.Tensor,
               stream: Optional[torch.cuda.Stream] = None) -> None:
        """Moves the accepted paths' rows behind the contexts, in every layer."""
        n = req.num_requests
        if accepted_node.dtype != torch.int32 or accepted_node.device != self.device or \
                accepted_node.dim() != 1 or accepted_node.shape[0] < n or not accepted_node.is_contiguous():
            raise ValueError("accepted_node is int32 [requests] on the pools' device")
        self._requests(n)
        with self._enter():
            B.check(self._lib.spec_cache_commit(req, self._ref, accepted_node.data_ptr(), self._stream(stream)),
                    "spec_cache_commit")

    def copy_pages(self, copies, stream: Optional[torch.cuda.Stream] = None) -> None:
        """Copies (src, dst, tokens) [n, 3], in every layer."""
        a = copies
        if not (isinstance(a, np.ndarray) and a.dtype == np.int32 and a.flags.c_contiguous):
            a = B.int32_copy(a)
        if a.size and (a.ndim != 2 or a.shape[1] != 3):
            raise ValueError("copies are [n, 3]: source, destination, tokens")
        with self._enter():
            B.check(self._lib.spec_cache_copy_pages(self._ref, a.ctypes.data if a.size else None, a.size // 3,
                                                    self._stream(stream)), "spec_cache_copy_pages")


class ChunkAttention(StagingRing):
    """Runs spec_chunk_attn on a PagedCache.  Owns a device workspace, which
    grows with the batches, and `ring` pinned staging buffers (StagingRing).  A
    graph is captured from B.spec_chunk_attn with a workspace and staging of its
    own: a replay reads the staging it was captured with, and here the ring
    reuses its slots, so a call on a capturing stream is refused.  An object is
    used by one thread at a time."""

    def __init__(self, cache: PagedCache, num_q_heads: int, scale: float = 0.0, ring: int = 32, event_every: int = 8):
        if event_every < 1 or ring < event_every:
            raise ValueError("need ring >= event_every >= 1")
        self.cache = cache
        a = self.args = B.SpecChunkAttnArgs()
        a.num_q_heads, a.scale = B.int32(num_q_heads), scale
        self._args_ref = C.byref(a)
        self._head = torch.Size((num_q_heads, cache.c.head_dim))
        self.ws_bytes = self.staging_bytes = 0
        self.ws_ptr = self._ws = self._pinned = None
        self._ring([None] * ring, event_every)
        _let_go()

    def __del__(self):
        # the last call may still read the staging and write the workspace, and
        # both go back to torch's allocators, which know of neither
        last = getattr(self, "_last_stream", None)
        if last is None:
            return
        try:
            _kept.append((last, self._ws, self._pinned))
            _let_go()
        except Exception:                     # the interpreter or the device is going away
            pass

    def _grow(self, chunks, stream) -> None:
        st, dev, host = B.spec_chunk_workspace_bytes(chunks, self.cache.c, self.args)
        B.check(st, "spec_chunk_workspace_bytes")
        if dev > self.ws_bytes:
            if self.ws_bytes:
                stream.synchronize()          # earlier calls' workspace goes back to the allocator
            self.ws_bytes = dev + dev // 4
            with torch.cuda.stream(stream):       # a block that no other stream's pending work has
                self._ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=self.cache.device)
            self.ws_ptr = (self._ws.data_ptr() + 255) // 256 * 256
        if host > self.staging_bytes:
            if self.staging_bytes:
                stream.synchronize()          # and their staging
            self.staging_bytes = host + host // 4
            size = (self.staging_bytes + 255) // 256 * 256
            self._pinned = torch.empty(size * len(self._staging), dtype=torch.uint8, pin_memory=True)
            self._staging = [self._pinned.data_ptr() + i * size for i in range(len(self._staging))]

    def run(self, chunks: B.SpecChunks, q: torch.Tensor, out: torch.Tensor, layer: int = 0,
            stream: Optional[torch.cuda.Stream] = None) -> None:
        """Attention of q [rows, Hq, d] into out [rows, Hq, d] (bf16 or fp32)."""
        cache, a = self.cache, self.args
        rows, head = chunks.rows, self._head
        qs, os, st = q.shape, out.shape, q.stride()
        if len(qs) != 3 or len(os) != 3 or qs[0] < rows or os[0] < rows or qs[1:] != head or os[1:] != head:
            raise ValueError("q and out are [rows, Hq, d], a row for every new token")
        kind = _DTYPE.get(out.dtype)
        if q.dtype != cache.dtype or kind is None or q.device != cache.device or out.device != cache.device or \
                not out.is_contiguous() or st[2] != 1:
            raise ValueError("q has the cache's type, out is contiguous bf16 or fp32, both on its device")
        cache._requests(chunks.num_requests)
        a.layer, a.out_dtype = B.int32(layer), kind
        a.q, a.out = q.data_ptr(), out.data_ptr()
        a.q_stride_tok = st[0] if qs[0] > 1 else qs[1] * qs[2]
        a.q_stride_head = st[1] if qs[1] > 1 else qs[2]
        with cache._enter():
            h = cache._stream(stream)
            if B.stream_capturing(h):
                raise RuntimeError("a graph's calls need a workspace and staging of their own: capture B.spec_chunk_attn")
            stream = stream or cache._streams[h]
            self._order(stream)
            for grown in (False, True):
                s = self._slot(stream)
                try:
                    st = cache._lib.spec_chunk_attn(chunks, cache._ref, self._args_ref, self.ws_ptr, self.ws_bytes,
                                                    self._staging[s], self.staging_bytes, h)
                finally:
                    self._done(s, stream)
                if st != B.SPEC_ERR_WORKSPACE or grown:
                    break
                self._grow(chunks, stream)
        B.check(st, "spec_chunk_attn")
