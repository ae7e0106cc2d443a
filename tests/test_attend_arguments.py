"""What the windowed and the shared attention refuse, and what their plans need,
on a host without a GPU."""
import os

import numpy as np
import pytest
import torch

from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention, PagedCache
from test_cache_abi import CHUNKS, FAKE, INV, UNS, WSP, _args, _cache


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_17074_amd import build
        build.build()
    return B.load()


def _window(w, sinks=0, chunks=None, cache=None, args=None, ws=FAKE, wsb=1 << 30, st=FAKE, stb=1 << 30):
    return B.spec_chunk_attn_window(chunks or B.make_chunks(*CHUNKS), cache or _cache(), args or _args(),
                                    None if w is None else B.SpecWindow(w, sinks), ws, wsb, st, stb, 0)


def _shared(groups, chunks=None, cache=None, args=None, ws=FAKE, wsb=1 << 30, st=FAKE, stb=1 << 30):
    return B.spec_chunk_attn_shared(chunks or B.make_chunks(*CHUNKS), cache or _cache(), args or _args(),
                                    groups and B.make_prefixes(*groups), ws, wsb, st, stb, 0)


@pytest.mark.parametrize("w,sinks", [(0, 0), (-1, 0), (5, -1), (-2**31, 0), (1, -2**31), (None, 0)])
def test_windows_refused(w, sinks):
    assert _window(w, sinks) == INV


CTX = ([10, 0, 300], [5, 64, 1])


@pytest.mark.parametrize("groups", [
    None,
    ([2], [0]),                            # a request is left over
    ([2, 2], [0, 0]),                      # one too many
    ([3, 1], [0, 0]), ([0, 3], [0, 0]), ([4, -1], [0, 0]), ([2**31 - 1], [0]),
    ([3], [1]),                            # request 1 has no context
    ([1, 2], [11, 0]), ([1, 1, 1], [0, 0, 301]), ([1, 1, 1], [-1, 0, 0]),
])
def test_prefixes_refused(groups):
    assert B.make_chunks(*CTX).rows == 70
    assert _shared(groups, chunks=B.make_chunks(*CTX)) == INV


def test_no_groups_and_no_arrays_are_refused():
    p = B.make_prefixes([3], [0])
    p.num_groups = 0
    call = lambda: B.spec_chunk_attn_shared(B.make_chunks(*CTX), _cache(), _args(), p, FAKE, 1 << 30, FAKE, 1 << 30, 0)  # noqa: E731
    assert call() == INV
    p.num_groups, p.group_size = 1, None
    assert call() == INV
    with pytest.raises(ValueError):
        B.make_prefixes([3], [0, 1])
    with pytest.raises(ValueError):
        B.make_prefixes([1.5], [0])


def test_a_request_without_new_tokens_may_be_shorter_than_its_prefix():
    n = B.make_chunks([10, 400, 300], [0, 1, 1])
    st, dev, host = B.spec_chunk_shared_workspace_bytes(n, _cache(), _args(), B.make_prefixes([3], [256]))
    assert st == B.SPEC_OK and dev > 0 and host > 0


@pytest.mark.parametrize("call", [lambda **kw: _window(64, 4, **kw), lambda **kw: _shared(([3], [0]), **kw)],
                         ids=["window", "shared"])
def test_what_the_plain_call_refuses(call):
    assert call(cache=_cache(dtype=B.SPEC_F32)) == UNS
    assert call(cache=_cache(head_dim=96, kv_stride_head=96)) == UNS
    assert call(args=_args(num_q_heads=7)) == INV
    assert call(args=_args(layer=2)) == INV
    assert call(args=_args(out=FAKE + 4)) == INV
    assert call(chunks=B.make_chunks([639, 0, 0], [2, 0, 0])) == INV
    assert call(ws=None) == WSP
    assert call(wsb=10) == WSP
    assert call(ws=FAKE + 16) == WSP
    assert call(stb=0) == WSP
    assert call(chunks=B.make_chunks([5, 5, 5], [0, 0, 0])) == B.SPEC_OK


def test_a_window_needs_less_room_than_all_rows():
    """One token over 30000 rows is cut into pieces over its window alone."""
    c = _cache(num_pages=1000, block_stride=500, layer_stride=1000 * 64 * 256)
    one = B.make_chunks([30000], [1])
    full = B.spec_chunk_workspace_bytes(one, c, _args())
    all_of_it = B.spec_chunk_window_workspace_bytes(one, c, _args(), B.SpecWindow(30001, 0))
    part = B.spec_chunk_window_workspace_bytes(one, c, _args(), B.SpecWindow(512, 4))
    assert full[0] == all_of_it[0] == part[0] == B.SPEC_OK
    assert full[1] == all_of_it[1] and part[1] < full[1]


def test_a_shared_prefix_is_planned_once():
    """Sixteen requests of a token behind 20000 rows: fewer pieces than for each alone."""
    c = _cache(num_pages=1000, block_stride=500, layer_stride=1000 * 64 * 256)
    n = B.make_chunks([20000] * 16, [1] * 16)
    full = B.spec_chunk_workspace_bytes(n, c, _args())
    once = B.spec_chunk_shared_workspace_bytes(n, c, _args(), B.make_prefixes([16], [20000]))
    assert full[0] == once[0] == B.SPEC_OK and once[2] < full[2]


def test_arguments_of_the_classes():
    k = torch.zeros((1, 4, 32, 2, 64), dtype=torch.bfloat16)
    cache = PagedCache(k, k.clone(), torch.zeros((2, 2), dtype=torch.int32))
    for kw in (dict(window=0), dict(window=-3), dict(window=5, sinks=-1), dict(sinks=4), dict(window=2**31)):
        with pytest.raises(ValueError):
            ChunkAttention(cache, 4, ring=8, **kw)
    att = ChunkAttention(cache, 4, window=7, sinks=2)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="window"):
        att.run(B.make_chunks([3], [2]), q, q.clone(), prefixes=B.make_prefixes([1], [0]))
    assert np.all(q.float().numpy() == 0)
