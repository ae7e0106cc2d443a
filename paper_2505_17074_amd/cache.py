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
# and to the current device, asked for only where tensors are on one
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


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
        self._head = tuple(k.shape[3:])
        self._width = k.shape[3] * k.shape[4]
        self._lib = B.load()
        c = self.c = B.SpecCache()
        self._ref = C.byref(c)
        self._append = B.SpecAppendArgs()
        self._append_ref = C.byref(self._append)
        self._rotation = B.SpecRotation()
        self._rotation_ref = C.byref(self._rotation)
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
        return _HERE if _current_device() == self._index else torch.cuda.device(self._index)

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

    def _new_rows(self, chunks: B.SpecChunks, k_new: torch.Tensor, v_new: torch.Tensor, layer: int) -> int:
        """The append arguments; the number of layers."""
        shape, st = k_new.shape, k_new.stride()
        if len(shape) not in (3, 4) or (v_new.shape != shape or v_new.stride() != st) and not _alike(k_new, v_new):
            raise ValueError("k_new and v_new are [layers, rows, Hkv, d], a row for every new token")
        if len(shape) == 4:
            (layers, rows, heads, d), (by_layer, by_row, by_head, by_one) = shape, st
        else:
            (rows, heads, d), (by_row, by_head, by_one) = shape, st
            layers, by_layer = 1, by_row
        if (heads, d) != self._head or rows < chunks.rows or (by_one != 1 and d > 1):
            raise ValueError("k_new and v_new are [layers, rows, Hkv, d], a row for every new token")
        dtype, device = self.dtype, self.device
        if k_new.dtype != dtype or v_new.dtype != dtype or k_new.device != device or v_new.device != device:
            raise ValueError("k_new and v_new have the pools' type and device")
        self._requests(chunks.num_requests)
        a = self._append
        a.layer, a.num_layers = B.int32(layer), layers
        a.k_new, a.v_new = k_new.data_ptr(), v_new.data_ptr()
        a.new_stride_layer = by_layer
        a.new_stride_tok = by_row if rows > 1 else self._width
        a.new_stride_head = by_head if heads > 1 else d
        return layers

    def append(self, chunks: B.SpecChunks, k_new: torch.Tensor, v_new: torch.Tensor, layer: int = 0,
               stream: Optional[torch.cuda.Stream] = None) -> None:
        """Rows k_new, v_new [layers, rows, Hkv, d] (or [rows, Hkv, d]: one layer)
        to the ends of the requests, in the cache's layers from `layer` on."""
        self._new_rows(chunks, k_new, v_new, layer)
        with self._enter():
            B.check(self._lib.spec_cache_append(chunks, self._ref, self._append_ref, self._stream(stream)),
                    "spec_cache_append")

    def _queries(self, q: torch.Tensor, rows: int):
        """Heads, address, and strides of a row and a head of queries."""
        shape = q.shape
        if len(shape) != 3:
            raise ValueError("q and q_out are [rows, Hq, d]")
        (n, heads, d), (by_row, by_head, by_one) = shape, q.stride()
        if n < rows or heads < 1 or d != self._head[1] or (by_one != 1 and d > 1):
            raise ValueError("q and q_out are [rows, Hq, d], a row for every new token")
        if q.dtype != self.dtype or q.device != self.device:
            raise ValueError("q and q_out have the pools' type and device")
        # of a dimension with one entry any stride will do
        return heads, q.data_ptr(), by_row if n > 1 else heads * d, by_head if heads > 1 else d

    def append_rotated(self, chunks: B.SpecChunks, k_new: torch.Tensor, v_new: torch.Tensor, freq: torch.Tensor,
                       q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                       positions: Optional[torch.Tensor] = None, interleaved: bool = False, layer: int = 0,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
        """append with K, and the queries q [rows, Hq, d] into q_out (or in place:
        q_out = q), turned by their positions on the way: pair i of a head's first
        2 len(freq) elements by position x freq[i] radians.  Pairs are elements i
        and i + len(freq), or, interleaved, 2 i and 2 i + 1.  freq is fp32;
        positions int32 [rows], without them a row's place in its request."""
        layers = self._new_rows(chunks, k_new, v_new, layer)
        rows, device = chunks.rows, self.device
        r = self._rotation
        shape = freq.shape
        if freq.dtype != torch.float32 or len(shape) != 1 or freq.device != device or \
                (shape[0] > 1 and freq.stride(0) != 1):
            raise ValueError("freq is fp32 [rotary dim / 2] on the pools' device")
        r.rotary_dim, r.interleaved, r.freq = 2 * shape[0], 1 if interleaved else 0, freq.data_ptr()
        if positions is None:
            r.positions = None
        else:
            shape = positions.shape
            if positions.dtype != torch.int32 or len(shape) != 1 or positions.device != device or shape[0] < rows or \
                    (shape[0] > 1 and positions.stride(0) != 1):
                raise ValueError("positions are int32 [rows] on the pools' device")
            r.positions = positions.data_ptr()
        if (q is None) != (q_out is None):
            raise ValueError("q and q_out go together")
        if q is None:
            r.num_q_heads = 0
        else:
            heads, r.q, r.q_stride_tok, r.q_stride_head = self._queries(q, rows)
            if q_out is q:
                r.q_out, r.out_stride_tok, r.out_stride_head = r.q, r.q_stride_tok, r.q_stride_head
            else:
                out_heads, r.q_out, r.out_stride_tok, r.out_stride_head = self._queries(q_out, rows)
                if out_heads != heads:
                    raise ValueError("q and q_out are [rows, Hq, d], a row for every new token")
            if layers != 1:
                raise ValueError("queries belong to one layer")
            r.num_q_heads = heads
        with self._enter():
            B.check(self._lib.spec_cache_append_rotated(chunks, self._ref, self._append_ref, self._rotation_ref,
                                                        self._stream(stream)), "spec_cache_append_rotated")

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
    """Runs spec_chunk_attn on a PagedCache; with `window`, spec_chunk_attn_window
    (a token sees the last `window` rows up to its own and the first `sinks`); a
    call with prefixes, spec_chunk_attn_shared.  Owns a device workspace, which
    grows with the batches, and `ring` pinned staging buffers (StagingRing).  A
    graph is captured from B.spec_chunk_attn with a workspace and staging of its
    own: a replay reads the staging it was captured with, and here the ring
    reuses its slots, so a call on a capturing stream is refused, and one on
    another stream while the last call's captures.  An object is used by one
    thread at a time."""

    def __init__(self, cache: PagedCache, num_q_heads: int, scale: float = 0.0, ring: int = 32, event_every: int = 8,
                 window: Optional[int] = None, sinks: int = 0):
        if event_every < 1 or ring < event_every:
            raise ValueError("need ring >= event_every >= 1")
        if window is None and sinks:
            raise ValueError("sinks belong to a window")
        self._window = None
        if window is not None:
            self._window = B.SpecWindow(B.int32(window), B.int32(sinks))
            if window < 1 or sinks < 0:
                raise ValueError("a window has at least a token's own row, sinks are not negative")
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

    def _grow(self, chunks, stream, prefixes) -> None:
        if self._window is not None:
            st, dev, host = B.spec_chunk_window_workspace_bytes(chunks, self.cache.c, self.args, self._window)
        elif prefixes is not None:
            st, dev, host = B.spec_chunk_shared_workspace_bytes(chunks, self.cache.c, self.args, prefixes)
        else:
            st, dev, host = B.spec_chunk_workspace_bytes(chunks, self.cache.c, self.args)
        B.check(st, "spec_chunk_workspace_bytes")
        if dev > self.ws_bytes:
            if self.ws_bytes:
                stream.synchronize()          # earlier calls' workspace goes back to the allocator
            size = dev + dev // 4
            with torch.cuda.stream(stream):       # a block that no other stream's pending work has
                ws = torch.empty(size + 256, dtype=torch.uint8, device=self.cache.device)
            # nothing raises from here on: the size is that of the memory at the address
            self._ws, self.ws_ptr, self.ws_bytes = ws, (ws.data_ptr() + 255) // 256 * 256, size
        if host > self.staging_bytes:
            if self.staging_bytes:
                stream.synchronize()          # and their staging
            slots, size = len(self._staging), host + host // 4
            apart = (size + 255) // 256 * 256
            pinned = torch.empty(apart * slots, dtype=torch.uint8, pin_memory=True)
            places = [pinned.data_ptr() + i * apart for i in range(slots)]
            self._pinned, self._staging, self.staging_bytes = pinned, places, size

    def run(self, chunks: B.SpecChunks, q: torch.Tensor, out: torch.Tensor, layer: int = 0,
            stream: Optional[torch.cuda.Stream] = None, prefixes: Optional[B.SpecPrefixes] = None) -> None:
        """Attention of q [rows, Hq, d] into out [rows, Hq, d] (bf16 or fp32).
        prefixes (B.make_prefixes): neighbouring requests that begin with the same
        rows, which are read once for all of them."""
        if prefixes is not None and self._window is not None:
            raise ValueError("shared prefixes have no window")
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
            self._not_into_a_graph(stream)
            self._order(stream)
            for grown in (False, True):
                s = self._slot(stream)
                try:
                    where = self.ws_ptr, self.ws_bytes, self._staging[s], self.staging_bytes, h
                    if self._window is not None:
                        st = cache._lib.spec_chunk_attn_window(chunks, cache._ref, self._args_ref, self._window, *where)
                    elif prefixes is not None:
                        st = cache._lib.spec_chunk_attn_shared(chunks, cache._ref, self._args_ref, prefixes, *where)
                    else:
                        st = cache._lib.spec_chunk_attn(chunks, cache._ref, self._args_ref, *where)
                finally:
                    self._done(s, stream)
                if st != B.SPEC_ERR_WORKSPACE or grown:
                    break
                self._grow(chunks, stream, prefixes)
        B.check(st, "spec_chunk_attn")
