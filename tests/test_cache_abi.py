"""The paged cache's entry points on a GPU-less host: every argument check,
which runs before the first HIP call, and the workspace sizes."""
import numpy as np
import pytest
import torch

from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention, PagedCache

FAKE = 1 << 20      # a 256-aligned fake device address; never dereferenced on these paths
INV, UNS, WSP = B.SPEC_ERR_INVALID_ARG, B.SPEC_ERR_UNSUPPORTED, B.SPEC_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_17074_amd import build
        build.build()
    return B.load()


def _cache(**kw):
    c = B.SpecCache()
    c.num_layers, c.num_kv_heads, c.head_dim, c.dtype = 2, 2, 128, B.SPEC_BF16
    c.num_pages, c.page_tokens = 100, 64
    c.k = c.v = c.block_table = FAKE
    c.kv_stride_tok, c.kv_stride_head = 256, 128
    c.layer_stride = 100 * 64 * 256
    c.block_stride = 10
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _args(**kw):
    a = B.SpecChunkAttnArgs()
    a.num_q_heads, a.out_dtype = 8, B.SPEC_BF16
    a.q = a.out = FAKE
    a.q_stride_tok, a.q_stride_head = 1024, 128
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _append(**kw):
    a = B.SpecAppendArgs()
    a.layer, a.num_layers = 0, 1
    a.k_new = a.v_new = FAKE
    a.new_stride_layer, a.new_stride_tok, a.new_stride_head = 1 << 20, 256, 128
    for k, v in kw.items():
        setattr(a, k, v)
    return a


CHUNKS = ([10, 0, 300], [5, 64, 1])


def _attn(chunks=None, cache=None, args=None, ws=FAKE, wsb=1 << 30, st=FAKE, stb=1 << 30):
    return B.spec_chunk_attn(chunks or B.make_chunks(*CHUNKS), cache or _cache(), args or _args(), ws, wsb, st, stb, 0)


BAD_CACHE = [
    (dict(num_layers=0), INV), (dict(num_kv_heads=0), INV), (dict(head_dim=0), INV), (dict(dtype=7), INV),
    (dict(num_pages=0), INV), (dict(page_tokens=0), INV), (dict(page_tokens=16), INV), (dict(page_tokens=48), INV),
    (dict(k=None), INV), (dict(v=None), INV), (dict(k=FAKE + 8), INV), (dict(v=FAKE + 2), INV),
    (dict(kv_stride_tok=0), INV), (dict(kv_stride_tok=-256), INV), (dict(kv_stride_tok=260), INV),
    (dict(kv_stride_tok=248), INV), (dict(kv_stride_head=64), INV), (dict(kv_stride_head=132), INV),
    (dict(kv_stride_head=1 << 33), INV), (dict(kv_stride_tok=1 << 33), INV),
    (dict(layer_stride=0), INV), (dict(layer_stride=12), INV),
    (dict(page_tokens=1 << 20, kv_stride_tok=1 << 12), UNS), (dict(num_layers=40000), UNS),
    (dict(head_dim=36, kv_stride_head=40, kv_stride_tok=80), UNS),
]
BAD_TABLE = [(dict(block_table=None), INV), (dict(block_table=FAKE + 2), INV), (dict(block_stride=0), INV),
             (dict(block_stride=4), INV)]


@pytest.mark.parametrize("kw,want", BAD_CACHE + BAD_TABLE)
def test_cache_refusals(kw, want):
    c, chunks = _cache(**kw), B.make_chunks(*CHUNKS)
    assert _attn(cache=c) == want
    assert B.spec_chunk_workspace_bytes(chunks, c, _args())[0] == want
    assert B.spec_cache_append(chunks, c, _append(), 0) == want
    assert B.spec_cache_commit(B.make_requests([10, 0, 300], None, [-1, 0, 0]), c, FAKE, 0) == want
    if (kw, want) in BAD_CACHE:
        one = np.array([[1, 2, 3]], np.int32)
        assert B.spec_cache_copy_pages(c, one.ctypes.data, 1, 0) == want


@pytest.mark.parametrize("ctx,new", [([-1], [5]), ([5], [-1]), ([640], [1]), ([0], [641]), ([2**31 - 1], [1]),
                                     ([0, 2**30], [1, 2**30])])
def test_length_refusals(ctx, new):
    chunks = B.make_chunks(ctx, new)
    assert _attn(chunks=chunks) == INV
    assert B.spec_cache_append(chunks, _cache(), _append(), 0) == INV


def test_null_arguments():
    chunks = B.make_chunks(*CHUNKS)
    assert B.spec_chunk_attn(None, _cache(), _args(), FAKE, 1 << 30, FAKE, 1 << 30, 0) == INV
    assert B.spec_chunk_attn(chunks, None, _args(), FAKE, 1 << 30, FAKE, 1 << 30, 0) == INV
    assert B.spec_chunk_attn(chunks, _cache(), None, FAKE, 1 << 30, FAKE, 1 << 30, 0) == INV
    assert B.load().spec_chunk_workspace_bytes(chunks, _cache(), _args(), None, None) == INV
    assert B.spec_cache_append(None, _cache(), _append(), 0) == INV
    assert B.spec_cache_append(chunks, None, _append(), 0) == INV
    assert B.spec_cache_append(chunks, _cache(), None, 0) == INV
    for field in ("ctx_len", "new_len"):
        broken = B.make_chunks(*CHUNKS)
        setattr(broken, field, None)
        assert _attn(chunks=broken) == INV
    empty = B.make_chunks([1], [1])
    empty.num_requests = 0
    assert _attn(chunks=empty) == INV


@pytest.mark.parametrize("kw,want", [
    (dict(num_q_heads=0), INV), (dict(num_q_heads=7), INV), (dict(layer=-1), INV), (dict(layer=2), INV),
    (dict(out_dtype=3), INV), (dict(q=None), INV), (dict(out=None), INV), (dict(q=FAKE + 4), INV),
    (dict(out=FAKE + 8), INV), (dict(q_stride_tok=0), INV), (dict(q_stride_tok=1028), INV),
    (dict(q_stride_head=-128), INV), (dict(q_stride_head=130), INV)])
def test_attention_refusals(kw, want):
    assert _attn(args=_args(**kw)) == want


def test_attention_types():
    assert _attn(cache=_cache(dtype=B.SPEC_F32)) == UNS
    assert _attn(cache=_cache(head_dim=96)) == UNS
    assert _attn(cache=_cache(head_dim=32)) == UNS


def test_attention_workspace():
    chunks = B.make_chunks([500, 0], [100, 30])
    st, dev, host = B.spec_chunk_workspace_bytes(chunks, _cache(), _args())
    assert st == B.SPEC_OK and dev >= host > 0
    for kw in (dict(ws=None), dict(ws=FAKE + 128), dict(wsb=dev - 1), dict(st=None), dict(stb=host - 1)):
        assert _attn(chunks=chunks, **kw) == WSP
    # nothing new: nothing to do, whatever the workspace
    assert _attn(chunks=B.make_chunks([5, 0], [0, 0]), ws=None, wsb=0, st=None, stb=0) == B.SPEC_OK


@pytest.mark.parametrize("kw", [
    dict(layer=-1), dict(layer=2), dict(num_layers=0), dict(num_layers=3), dict(layer=1, num_layers=2),
    dict(num_layers=2**31 - 1), dict(k_new=None), dict(v_new=None), dict(k_new=FAKE + 8), dict(v_new=FAKE + 2),
    dict(new_stride_tok=0), dict(new_stride_tok=260), dict(new_stride_head=0), dict(new_stride_head=129),
    dict(num_layers=2, new_stride_layer=0), dict(num_layers=2, new_stride_layer=4)])
def test_append_refusals(kw):
    assert B.spec_cache_append(B.make_chunks(*CHUNKS), _cache(), _append(**kw), 0) == INV


def test_append_of_nothing():
    assert B.spec_cache_append(B.make_chunks([7, 2000], [0, 0]), _cache(), _append(k_new=None, v_new=None), 0) == B.SPEC_OK


def test_commit_refusals():
    c = _cache()
    req = B.make_requests([10, 20], None, [-1, 0, 0])
    assert B.spec_cache_commit(None, c, FAKE, 0) == INV
    assert B.spec_cache_commit(req, None, FAKE, 0) == INV
    assert B.spec_cache_commit(req, c, None, 0) == INV
    assert B.spec_cache_commit(req, c, FAKE + 2, 0) == INV
    for ctx, kw in (([-1], dict(tree_parent=[-1, 0])), ([639], dict(tree_parent=[-1, 0])),
                    ([1], dict(tree_parent=[0, 0])), ([1], dict(tree_parent=[-1, 1])), ([1], dict(tree_parent=[-1, -1])),
                    ([1], dict(tree_parent=[-1] + [0] * 32)), ([1], dict(tree_parents=[[-1, 0, 2]])),
                    ([639, 0], dict(tree_parents=[[-1, 0], [-1]])), ([1], dict(draft_len=[17])), ([1], dict(draft_len=[-1])),
                    ([1], dict())):
        assert B.spec_cache_commit(B.make_requests(ctx, **kw), c, FAKE, 0) == INV, (ctx, kw)
    both = B.make_requests([1], tree_parents=[[-1, 0]])
    both.tree_nodes = 2
    assert B.spec_cache_commit(both, c, FAKE, 0) == INV
    # chains are in place: accepted without a launch
    assert B.spec_cache_commit(B.make_requests([10, 20], [3, 0]), c, FAKE, 0) == B.SPEC_OK


@pytest.mark.parametrize("copies", [
    [[-1, 2, 3]], [[100, 2, 3]], [[1, -1, 3]], [[1, 100, 3]], [[1, 2, 0]], [[1, 2, 65]], [[1, 1, 3]],
    [[1, 2, 3], [5, 2, 3]], [[1, 2, 3], [2, 4, 3]], [[4, 2, 3], [1, 4, 3]]])
def test_copy_refusals(copies):
    a = np.array(copies, np.int32)
    assert B.spec_cache_copy_pages(_cache(), a.ctypes.data, len(copies), 0) == INV
    assert B.spec_cache_copy_pages(_cache(), None, 1, 0) == INV
    assert B.spec_cache_copy_pages(_cache(), a.ctypes.data, -1, 0) == INV


def test_copy_of_nothing():
    assert B.spec_cache_copy_pages(_cache(block_table=None), None, 0, 0) == B.SPEC_OK


def test_python_refusals():
    """The tensors' shapes, types and places, checked before the library is called."""
    k, v = torch.zeros((1, 4, 32, 2, 64)), torch.zeros((1, 4, 32, 2, 64))
    t = torch.zeros((2, 2), dtype=torch.int32)
    for a, b in ((k[0], v[0]), (k, v[..., :32]), (k, v.bfloat16()), (k.half(), v.half()), (k, v.transpose(2, 3)),
                 (k[:, :, :16], v[:, :, :16])):
        with pytest.raises(ValueError):
            PagedCache(a, b, t)
    for bad in (t.long(), t[0], t.t()[:, :1].expand(2, 2)):
        with pytest.raises(ValueError):
            PagedCache(k, v, bad)
    c = PagedCache(k, v, t)
    chunks = B.make_chunks([0, 0], [3, 2])
    rows = torch.zeros((5, 2, 64))
    for kk, vv in ((rows[:4], rows[:4]), (rows, rows[:, :1]), (rows.bfloat16(), rows.bfloat16()), (rows[..., :32], rows[..., :32])):
        with pytest.raises(ValueError):
            c.append(chunks, kk, vv)
    with pytest.raises(ValueError):
        c.append(B.make_chunks([0] * 3, [1] * 3), rows, rows)          # three requests, two rows of the table
    with pytest.raises(ValueError):
        c.commit(B.make_requests([0, 0], None, [-1, 0]), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        c.commit(B.make_requests([0, 0], None, [-1, 0]), torch.zeros(1, dtype=torch.int32))
    kb = k.bfloat16()
    att = ChunkAttention(PagedCache(kb, kb.clone(), t), 4)
    q, o = torch.zeros((5, 4, 64), dtype=torch.bfloat16), torch.zeros((5, 4, 64))
    for qq, oo in ((q[:4], o), (q, o[:4]), (q.float(), o), (q, o.half()), (q[:, :2], o), (q, o.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            att.run(chunks, qq, oo)
    with pytest.raises(ValueError):
        B.make_chunks([1, 2], [1])


def test_pools_in_host_memory():
    """Every call on pools that no GPU holds is refused before the library sees it."""
    k = torch.zeros((1, 4, 32, 2, 64), dtype=torch.bfloat16)
    c = PagedCache(k, k.clone(), torch.zeros((2, 2), dtype=torch.int32))
    chunks, rows = B.make_chunks([0, 0], [3, 2]), torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    q, o = torch.zeros((5, 4, 64), dtype=torch.bfloat16), torch.zeros((5, 4, 64))
    for call in (lambda: c.append(chunks, rows, rows), lambda: c.copy_pages([(0, 1, 3)]),
                 lambda: c.commit(B.make_requests([0, 0], None, [-1, 0]), torch.zeros(2, dtype=torch.int32)),
                 lambda: ChunkAttention(c, 4).run(chunks, q, o)):
        with pytest.raises(ValueError, match="device memory"):
            call()


def test_strides_of_single_entries():
    """A dimension of one entry may have any stride, and K and V different ones."""
    k = torch.zeros((4, 32, 2, 64)).as_strided((1, 4, 32, 2, 64), (7, 4096, 128, 64, 1))
    v = torch.zeros((1, 4, 32, 2, 64))
    c = PagedCache(k, v, torch.zeros((2, 5), dtype=torch.int32)[:, :1])
    assert (c.c.kv_stride_tok, c.c.kv_stride_head, c.c.block_stride) == (128, 64, 5)
    c.table = torch.zeros(2, dtype=torch.int32).as_strided((2, 1), (1, 3))
    with pytest.raises(ValueError, match="device memory"):             # and not their strides
        c.append(B.make_chunks([3], [1]), torch.zeros((1, 2, 64)), torch.zeros((1, 9, 64))[:, :2])
    with pytest.raises(ValueError, match="a row for every new token"):
        c.append(B.make_chunks([3], [2]), torch.zeros((2, 2, 64)), torch.zeros((2, 9, 64))[:, :2])


def test_more_copies_than_pages():
    """Refused before anything as long as the list is read."""
    assert B.spec_cache_copy_pages(_cache(), np.zeros(3, np.int32).ctypes.data, 2**31 - 1, 0) == INV


def test_lengths_are_copied_and_whole():
    ctx, new = np.array([4, 5], np.int32), np.array([1, 2], np.int32)
    chunks = B.make_chunks(ctx, new)
    ctx += 100
    new += 100
    assert [chunks.ctx_len[i] for i in range(2)] == [4, 5] and [chunks.new_len[i] for i in range(2)] == [1, 2]
    assert chunks.rows == 3
    for bad in ([1.5, 2], np.array([2**32, 1]), np.array([1, np.nan])):
        with pytest.raises(ValueError):
            B.make_chunks(bad, [1, 1])
        with pytest.raises(ValueError):
            B.make_chunks([1, 1], bad)
    k = torch.zeros((1, 4, 32, 2, 64))
    for bad in ([(0, 1, 2.5)], np.array([[2**32, 1, 3]])):
        with pytest.raises(ValueError, match="whole numbers"):
            PagedCache(k, k.clone()).copy_pages(bad)
