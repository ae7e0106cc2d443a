"""A workspace that cannot grow, on a host without a GPU: the allocation raises
and the object goes on with what it had, its sizes those of its memory."""
import os

import pytest
import torch

from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.sample import Sampler

FAKE = 1 << 20      # a fake device address; never dereferenced on these paths


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_17074_amd import build
        build.build()
    return B.load()


def _no_memory(*args, **kwargs):
    raise torch.OutOfMemoryError("no memory")


def _holds(tensor, ptr, size):
    """`size` bytes from ptr on are the tensor's."""
    return tensor.data_ptr() <= ptr and ptr + size <= tensor.data_ptr() + tensor.numel()


def _sampler():
    s = Sampler("cpu")
    a = s._args
    a.num_rows, a.vocab, a.dtype = 1, 1000, B.SPEC_F32
    a.logits = a.uniforms = a.tokens = FAKE
    s._grow()
    return s


def test_a_sampler_that_cannot_grow(monkeypatch):
    s = _sampler()
    held = s._ws, s._ws_ptr, s._ws_bytes
    assert _holds(*held)
    s._args.vocab = 1 << 20
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", _no_memory)
        with pytest.raises(torch.OutOfMemoryError):
            s._grow()
    assert s._ws is held[0] and (s._ws_ptr, s._ws_bytes) == held[1:]
    # so that the larger batch is still refused by the library's own check
    assert B.spec_sample(s._args, s._ws_ptr, s._ws_bytes, 0) == B.SPEC_ERR_WORKSPACE
    s._grow()
    assert s._ws is not held[0] and s._ws_bytes > held[2] and _holds(s._ws, s._ws_ptr, s._ws_bytes)
