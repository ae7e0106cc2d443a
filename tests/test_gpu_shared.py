"""GPU: attention of requests behind shared prefixes against the definition in
64 bits of each request alone.  Every place of the pools that no request owns is
NaN."""
import numpy as np
import pytest
import torch

from attend_util import causal_seen, reference
from cache_util import BF16, F32, Paged, check_close, queries
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention

pytestmark = pytest.mark.gpu

CASES = {
    # name: groups' sizes and prefixes, rows of their own, new, query heads, KV heads, d, page tokens
    "two_decode": ([2], [256], [3, 0], [1, 1], 8, 2, 128, 64),
    "answers": ([8], [1500], [5, 60, 0, 1, 31, 32, 33, 64], [1] * 8, 32, 8, 128, 64),
    "many_decode": ([40], [700], list(range(40)), [1] * 40, 8, 2, 128, 32),
    "rows_low": ([4], [300], [5, 6, 7, 8], [2, 1, 3, 2], 4, 1, 64, 32),
    "short_prefixes": ([3, 2, 2], [0, 63, 127], [5, 6, 7, 100, 3, 0, 9], [2, 1, 3, 2, 5, 70, 2], 8, 2, 128, 32),
    "prefix_edges": ([2, 2, 2, 2], [128, 129, 191, 192], [1, 2] * 4, [3, 40] * 4, 8, 2, 128, 32),
    "groups_and_single": ([3, 1, 4, 1], [400, 900, 333, 0], [7, 0, 90, 30, 1, 2, 3, 4, 5], [1, 33, 4, 9, 1, 1, 70, 1, 2],
                          8, 2, 128, 64),
    "first_without_rows": ([3, 2], [500, 200], [0, 10, 20, 0, 4], [0, 5, 1, 0, 3], 8, 2, 128, 96),
    "one_with_rows": ([3], [500], [0, 10, 20], [0, 5, 0], 8, 2, 128, 96),
    "chunks_d64": ([5, 6], [1000, 640], [0] * 11, [10, 200, 33, 64, 1, 90, 128, 17, 5, 60, 100], 16, 4, 64, 96),
    "tiles_across_requests": ([3], [512], [0, 40, 9], [50, 100, 77], 12, 4, 128, 32),
    "wide_group": ([4], [600], [3, 2, 1, 0], [9, 1, 1, 30], 40, 1, 64, 160),
    "long_prefix": ([3], [9000], [100, 50, 2000], [1, 2, 1], 8, 1, 128, 256),
}


def make(sizes, prefixes, own, new, hkv, d, page, seed, layers=1, **kw):
    """Forked requests: a group's whole pages of the prefix are shared, the partly
    filled one copied."""
    prefix = np.repeat(prefixes, sizes)
    p = Paged(prefix + np.asarray(own), new, hkv, d, page, seed=seed, layers=layers, **kw)
    at = 0
    for n, m in zip(sizes, prefixes):
        for i in range(at + 1, at + n):
            p.table_np[i, :m // page] = p.table_np[at, :m // page]
            for x, first in zip(p.rows[i], p.rows[at]):
                x[:, :m] = first[:, :m]
        at += n
    p.table = torch.from_numpy(p.table_np).to(p.device)
    p.cache.table = p.table
    return p


def _run(p, q, out_dtype, prefixes, scale=0.0, layer=0):
    out = torch.full((q.shape[0] + 3, q.shape[1], q.shape[2]), 7.0, dtype=out_dtype, device="cuda")
    ChunkAttention(p.cache, q.shape[1], scale).run(p.chunks(), q.cuda(), out, layer=layer, prefixes=prefixes)
    torch.cuda.synchronize()
    assert (out[q.shape[0]:] == 7.0).all()               # rows past the last new token
    return out[:q.shape[0]]


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("name", CASES)
def test_matches_the_definition(gpu_lib, name, out):
    sizes, prefixes, own, new, hq, hkv, d, page = CASES[name]
    print(f"[case] shared {name} {out}", flush=True)
    p = make(sizes, prefixes, own, new, hkv, d, page, seed=len(name)).write()
    q = queries(sum(new), hq, d, seed=len(name))
    check_close(_run(p, q, out, B.make_prefixes(sizes, prefixes)), *reference(p, q, causal_seen(p), out=out))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [100, 450])
def test_values_that_are_not_finite(gpu_lib, at, bad):
    """In the prefix they reach all of its group and no other; in a request's own
    rows itself."""
    print(f"[case] shared not finite {at} {bad}", flush=True)
    p = make([2, 2], [400, 300], [100, 100, 50, 60], [3, 40, 5, 1], 2, 128, 32, seed=3)
    p.rows[0][1][:, at] = bad
    if at < 400:
        p.rows[1][1][:, at] = bad
    p.write()
    q = queries(49, 8, 128, seed=2)
    ref, bound = reference(p, q, causal_seen(p), out=F32)
    check_close(_run(p, q, F32, B.make_prefixes([2, 2], [400, 300])), ref, bound)
    assert np.isfinite(ref).all((1, 2)).tolist() == [False] * 3 + [at >= 400] * 40 + [True] * 6


def test_only_the_first_requests_pages_hold_the_prefix(gpu_lib):
    """The others' ids of the prefix's pages are not read where it is shared."""
    print("[case] shared ids", flush=True)
    p = make([3], [256], [9, 8, 7], [2, 30, 1], 2, 128, 64, seed=4).write()
    gone = p.table.clone()
    gone[1:, :4] = 1 << 29
    p.cache.table = gone
    q = queries(33, 4, 128, seed=2)
    check_close(_run(p, q, BF16, B.make_prefixes([3], [256])), *reference(p, q, causal_seen(p)))


def test_nothing_shared_is_the_plain_call(gpu_lib):
    print("[case] shared nothing", flush=True)
    p = Paged([1500, 3, 260], [1, 300, 40], 2, 128, seed=8).write()
    q = queries(341, 8, 128, seed=8).cuda()
    plain, out = (torch.empty((341, 8, 128), dtype=BF16, device="cuda") for _ in range(2))
    att = ChunkAttention(p.cache, 8)
    att.run(p.chunks(), q, plain)
    att.run(p.chunks(), q, out, prefixes=B.make_prefixes([1, 1, 1], [1000, 3, 0]))
    torch.cuda.synchronize()
    assert torch.equal(plain, out)


def test_scale_a_later_layer_and_strided_queries(gpu_lib):
    print("[case] shared strides", flush=True)
    p = make([2, 3], [200, 333], [4, 90, 2, 0, 1], [3, 64, 1, 2, 40], 2, 64, 32, seed=5, layers=3, gap=16).write()
    wide = torch.full((111, 10, 72), float("nan"), dtype=BF16, device="cuda")
    q = queries(110, 6, 64, seed=9)
    wide[:110, 2:8, :64] = q.cuda()
    out = torch.empty((110, 6, 64), dtype=F32, device="cuda")
    ChunkAttention(p.cache, 6, 0.3).run(p.chunks(), wide[:, 2:8, :64], out, layer=2,
                                        prefixes=B.make_prefixes([2, 3], [200, 333]))
    check_close(out, *reference(p, q, causal_seen(p), layer=2, scale=0.3, out=F32))


def test_captured_and_repeated(gpu_lib):
    print("[case] shared replay", flush=True)
    sizes, prefixes = [3, 4], [640, 999]
    p = make(sizes, prefixes, [5, 0, 60, 9, 9, 1, 2], [1, 40, 3, 1, 1, 7, 90], 2, 128, 64, seed=12).write()
    q = queries(143, 8, 128, seed=12).cuda()
    att = ChunkAttention(p.cache, 8)
    first, out = (torch.empty((143, 8, 128), dtype=BF16, device="cuda") for _ in range(2))
    chunks, groups = p.chunks(), B.make_prefixes(sizes, prefixes)
    att.run(chunks, q, first, prefixes=groups)
    a = B.SpecChunkAttnArgs()
    a.num_q_heads, a.out_dtype, a.q, a.out = 8, B.SPEC_BF16, q.data_ptr(), out.data_ptr()
    a.q_stride_tok, a.q_stride_head = 1024, 128
    st, dev, host = B.spec_chunk_shared_workspace_bytes(chunks, p.cache.c, a, groups)
    assert st == B.SPEC_OK
    ws = torch.empty(dev + 256, dtype=torch.uint8, device="cuda")
    staging = torch.empty(host, dtype=torch.uint8, pin_memory=True)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        B.check(B.spec_chunk_attn_shared(chunks, p.cache.c, a, groups, (ws.data_ptr() + 255) // 256 * 256, dev,
                                         staging.data_ptr(), host, stream.cuda_stream), "shared")
    other = torch.empty_like(first)
    for i in range(4):
        out.fill_(9.0)
        graph.replay()
        att.run(chunks, q, other, stream=None if i % 2 else stream, prefixes=groups)
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(other, first)


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("sizes,prefixes", [([20], [1000]), ([12, 9, 1], [640, 1500, 300])])
def test_single_tokens_of_small_heads(gpu_lib, sizes, prefixes, out):
    """d = 64: a prefix's rows fill tall tiles, each request's own one row of one."""
    print(f"[case] shared single d64 {sizes} {out}", flush=True)
    n = sum(sizes)
    p = make(sizes, prefixes, [(7 * i) % 150 for i in range(n)], [1] * n, 4, 64, 64, seed=n).write()
    q = queries(n, 16, 64, seed=n)
    check_close(_run(p, q, out, B.make_prefixes(sizes, prefixes)), *reference(p, q, causal_seen(p), out=out))
