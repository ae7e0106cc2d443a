"""A workspace that cannot grow, on a host without a GPU: the allocation raises
and the object goes on with what it had, its sizes those of its memory."""
import os

import pytest
import torch

from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention, PagedCache
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


class _Stream:
    """Stands for a device's stream: nothing is pending on it."""

    def synchronize(self):
        pass


def _prefixes(kind, n):
    return B.make_prefixes([n], [256]) if kind == "prefixes" else None


def _attention(kind):
    k = torch.zeros((1, 4, 32, 2, 64), dtype=torch.bfloat16)
    cache = PagedCache(k, k.clone(), torch.zeros((64, 4096), dtype=torch.int32))
    a = ChunkAttention(cache, 4, window=500 if kind == "window" else None, ring=4, event_every=2)
    a.args.q = a.args.out = FAKE
    a.args.q_stride_tok, a.args.q_stride_head = 256, 64
    return a


def _state(a):
    return a.ws_ptr, a.ws_bytes, a.staging_bytes, list(a._staging)


def _consistent(a):
    size = (a.staging_bytes + 255) // 256 * 256
    assert _holds(a._ws, a.ws_ptr, a.ws_bytes)
    assert _holds(a._pinned, a._staging[0], size * len(a._staging))
    assert [x - a._staging[0] for x in a._staging] == [i * size for i in range(len(a._staging))]


@pytest.mark.parametrize("fails", ["workspace", "staging"])
@pytest.mark.parametrize("kind", ["plain", "window", "prefixes"])
def test_an_attention_that_cannot_grow(monkeypatch, kind, fails):
    small = B.make_chunks([300, 300], [1, 1])
    large = B.make_chunks([90000] * 40, [900] * 40)        # its plan alone outgrows the first workspace
    empty = torch.empty
    broken = []

    def allocate(*size, pin_memory=False, **kw):
        if broken and pin_memory == (fails == "staging"):
            raise torch.OutOfMemoryError("no memory")
        return empty(*size, **kw)

    monkeypatch.setattr(torch, "empty", allocate)
    a = _attention(kind)
    a._grow(small, _Stream(), _prefixes(kind, 2))
    _consistent(a)
    was = _state(a)
    broken.append(True)
    with pytest.raises(torch.OutOfMemoryError):
        a._grow(large, _Stream(), _prefixes(kind, 40))
    now = _state(a)
    assert now[2:] == was[2:]
    if fails == "workspace":
        assert now == was
    _consistent(a)
    broken.clear()
    a._grow(large, _Stream(), _prefixes(kind, 40))
    assert a.ws_bytes > was[1] and a.staging_bytes > was[2]
    _consistent(a)
