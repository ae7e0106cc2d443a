"""Sampling (specsample.h): tokens from logits and given uniforms, and the
distributions they were drawn from.  Argument marshalling only; it runs in the
library's HIP kernels.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional

import torch

from . import binding as B
from .cache import _current_device, _current_raw_stream

_DTYPE = {torch.bfloat16: B.SPEC_BF16, torch.float32: B.SPEC_F32}
_HERE = contextlib.nullcontext()


class Sampler:
    """Runs spec_sample on one device.  Owns a device workspace, which grows with
    the batches.  Calls are serialised: one on another stream than the last waits
    for it.  A graph is captured from B.spec_sample with a workspace of its own: a
    replay would write this one beside later calls, so a call on a capturing stream
    is refused, and one on another stream while the last call's captures.  An object
    is used by one thread at a time.

    A call runs on `stream`, or the current one, after what is on it already; its
    tensors are its caller's to order and to keep, as for any work on a stream
    that is not their own."""

    def __init__(self, device="cuda"):
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._lib = B.load()
        self._args = B.SpecSampleArgs()
        self._ref = C.byref(self._args)
        self._ws = self._ws_ptr = None
        self._ws_bytes = 0
        self._last = self._last_h = None       # the last call's stream

    def _move(self, h: int, stream: torch.cuda.Stream) -> None:
        """The next call runs on another stream than the last, whose use of the
        workspace it waits for."""
        if self._last is not None:
            if B.stream_capturing(self._last_h):
                # an event there belongs to the graph, and who waits for it does so too
                raise RuntimeError("the last call's stream is capturing a graph, which would take this call in")
            stream.wait_event(self._last.record_event())
        if self._ws is not None:
            self._ws.record_stream(stream)
        self._last, self._last_h = stream, h

    def _grow(self) -> None:
        st, need = B.spec_sample_workspace_bytes(self._args)
        B.check(st, "spec_sample_workspace_bytes")
        # the last one goes back to torch's allocator, which knows the streams it was used on
        size = need + need // 4
        with torch.cuda.stream(self._last):    # a block that no other stream's pending work has
            ws = torch.empty(size + 256, dtype=torch.uint8, device=self.device)
        # nothing raises from here on: the size is that of the memory at the address
        self._ws, self._ws_ptr, self._ws_bytes = ws, (ws.data_ptr() + 255) // 256 * 256, size

    def _per_row(self, t: Optional[torch.Tensor], name: str, dtype: torch.dtype, rows: int) -> Optional[int]:
        if t is None:
            return None
        shape = t.shape
        if t.dtype != dtype or len(shape) != 1 or shape[0] != rows or t.device != self.device or \
                (rows > 1 and t.stride(0) != 1):
            raise ValueError(f"{name} is {dtype} [rows] on the sampler's device")
        return t.data_ptr()

    def run(self, logits: torch.Tensor, uniforms: Optional[torch.Tensor] = None, tokens: Optional[torch.Tensor] = None,
            temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
            top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None,
            probs: Optional[torch.Tensor] = None, kept_logits: Optional[torch.Tensor] = None,
            stream: Optional[torch.cuda.Stream] = None) -> None:
        """A token of each row of logits [rows, vocab] (bf16 or fp32) into tokens
        (int32 [rows]) by uniforms (fp32 [rows] in [0, 1)).  temperature, top_p and
        min_p are fp32 [rows], top_k int32 [rows]; without one there is no limit (and
        the temperature is 1).  probs: the distributions that the tokens were drawn
        from; kept_logits in its place: the logits of those distributions.  Both
        are [rows, vocab] of the logits' type and may be the logits themselves."""
        kind, shape = _DTYPE.get(logits.dtype), logits.shape
        if len(shape) != 2 or kind is None or logits.device != self.device or shape[0] < 1 or shape[1] < 1 or \
                (shape[1] > 1 and logits.stride(1) != 1):
            raise ValueError("logits are bf16 or fp32 [rows, vocab] on the sampler's device")
        if probs is not None and kept_logits is not None:
            raise ValueError("probs or kept_logits, not both")
        if tokens is not None and uniforms is None:
            raise ValueError("tokens need uniforms")
        n, vocab = shape
        a = self._args
        a.num_rows, a.vocab, a.dtype = B.int32(n), B.int32(vocab), kind
        a.logits, a.logits_stride = logits.data_ptr(), logits.stride(0) if n > 1 else vocab
        a.temperature = self._per_row(temperature, "temperature", torch.float32, n)
        a.top_k = self._per_row(top_k, "top_k", torch.int32, n)
        a.top_p = self._per_row(top_p, "top_p", torch.float32, n)
        a.min_p = self._per_row(min_p, "min_p", torch.float32, n)
        a.uniforms = self._per_row(uniforms, "uniforms", torch.float32, n)
        a.tokens = self._per_row(tokens, "tokens", torch.int32, n)
        rows = probs if probs is not None else kept_logits
        a.rows, a.rows_stride, a.rows_kind = None, 0, B.SPEC_SAMPLE_NONE
        if rows is not None:
            if rows.shape != logits.shape or rows.dtype != logits.dtype or rows.device != self.device or \
                    (vocab > 1 and rows.stride(1) != 1):
                raise ValueError("probs and kept_logits are [rows, vocab] of the logits' type and device")
            a.rows, a.rows_stride = rows.data_ptr(), rows.stride(0) if n > 1 else vocab
            a.rows_kind = B.SPEC_SAMPLE_PROBS if probs is not None else B.SPEC_SAMPLE_LOGITS
        if self.device.type != "cuda":
            raise ValueError("the logits are not in device memory")
        index = self.device.index
        with _HERE if _current_device() == index else torch.cuda.device(self.device):
            h = _current_raw_stream(index) if stream is None else stream.cuda_stream
            if B.stream_capturing(h):
                raise RuntimeError("a graph's calls need a workspace of their own: capture B.spec_sample")
            if h != self._last_h:
                self._move(h, stream or torch.cuda.current_stream(index))
            st = self._lib.spec_sample(self._ref, self._ws_ptr, self._ws_bytes, h)
            if st == B.SPEC_ERR_WORKSPACE:
                self._grow()
                st = self._lib.spec_sample(self._ref, self._ws_ptr, self._ws_bytes, h)
        B.check(st, "spec_sample")
