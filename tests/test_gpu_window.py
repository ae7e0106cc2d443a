"""GPU: attention with a sliding window and sinks over a paged cache against its
definition in 64 bits.  Every place of the pools that no request owns is NaN."""
import numpy as np
import pytest
import torch

from attend_util import reference, window_seen
from cache_util import BF16, F32, Paged, check_close, queries
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention

pytestmark = pytest.mark.gpu

CASES = {
    # name: ctx, new, query heads, KV heads, d, page tokens, window, sinks
    "first_token": ([0], [1], 4, 4, 128, 32, 1, 0),
    "own_row_alone": ([0, 5, 64, 300], [40, 3, 1, 70], 8, 2, 128, 64, 1, 0),
    "own_row_and_a_sink": ([0, 5, 64, 300], [40, 3, 1, 70], 8, 2, 128, 64, 1, 1),
    "one_token_each": ([0, 1, 31, 32, 63, 64, 65, 700], [1] * 8, 8, 2, 128, 32, 33, 4),
    "decode_long": ([5000, 1023, 2048], [1, 1, 1], 8, 1, 128, 64, 500, 4),
    "decode_cut": ([9000], [1], 32, 8, 128, 64, 4096, 4),
    "few_tokens": ([100, 0, 37], [3, 8, 5], 8, 2, 64, 64, 32, 0),
    "prompt": ([0], [333], 8, 2, 128, 64, 64, 3),
    "prompt_edges": ([0], [400], 4, 1, 128, 32, 65, 32),
    "prompt_mha": ([0, 0], [65, 128], 4, 4, 64, 96, 20, 33),
    "chunk_after_context": ([500, 77], [200, 129], 8, 2, 128, 96, 127, 64),
    "group_of_three": ([90, 10], [50, 43], 12, 4, 128, 32, 31, 5),
    "wide_group": ([300], [37], 40, 1, 64, 160, 100, 1),
    "with_nothing_new": ([40, 100, 7, 9], [0, 60, 0, 33], 8, 2, 128, 64, 17, 2),
    "mixed": ([1500, 3, 260, 0, 900], [1, 300, 1, 64, 31], 8, 2, 128, 64, 200, 4),
    "long_cut": ([6000], [40], 8, 2, 128, 256, 3000, 100),
    "long_many_tiles": ([700], [1500], 4, 2, 128, 64, 1000, 4),
    "sinks_behind_the_end": ([40, 500], [30, 30], 4, 2, 128, 32, 10, 200),
    "all_sinks": ([40, 300], [30, 5], 4, 2, 128, 32, 10, 100000),
    "window_past_the_start": ([40, 300, 2000], [30, 5, 200], 4, 2, 64, 32, 2**31 - 1, 3),
    "sinks_cut_off": ([3000], [100], 4, 2, 128, 64, 100, 1000),
}


def _run(p, q, out_dtype, window, sinks, scale=0.0, layer=0):
    out = torch.full((q.shape[0] + 3, q.shape[1], q.shape[2]), 7.0, dtype=out_dtype, device="cuda")
    att = ChunkAttention(p.cache, q.shape[1], scale, window=window, sinks=sinks)
    att.run(p.chunks(), q.cuda(), out, layer=layer)
    torch.cuda.synchronize()
    assert (out[q.shape[0]:] == 7.0).all()               # rows past the last new token
    return out[:q.shape[0]]


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("name", CASES)
def test_matches_the_definition(gpu_lib, name, out):
    ctx, new, hq, hkv, d, page, window, sinks = CASES[name]
    print(f"[case] window {name} {out}", flush=True)
    p = Paged(ctx, new, hkv, d, page, seed=len(name)).write()
    q = queries(sum(new), hq, d, seed=len(name))
    check_close(_run(p, q, out, window, sinks), *reference(p, q, window_seen(p, window, sinks), out=out))


def _out_of_sight(p, i, window, sinks):
    """Rows of request i that no new token sees."""
    return np.nonzero(~window_seen(p, window, sinks)(i).any(0))[0]


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 6, 90])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_out_of_sight_hold_anything(gpu_lib, new, out, d):
    """NaN and infinities in rows behind the window, and page ids there that are
    outside the pool or another's."""
    window, sinks = 70, 5
    print(f"[case] window out of sight {new} {out} {d}", flush=True)
    p = Paged([500, 333], [new, new], 2, d, page=32, seed=6)
    for i in range(2):
        far = _out_of_sight(p, i, window, sinks)
        assert far.size > 200
        for x, bad in zip(p.rows[i], (float("nan"), float("inf"))):
            x[:, far] = bad
    p.write()
    gone = p.table.clone()
    gone[0, 1:(500 - window) // 32] = 1 << 30
    gone[1, 1:(333 - window) // 32] = -5
    p.cache.table = gone
    q = queries(2 * new, 4, d, seed=1)
    check_close(_run(p, q, out, window, sinks), *reference(p, q, window_seen(p, window, sinks), out=out))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [2, 130, 200])
def test_a_row_reaches_those_that_see_it(gpu_lib, at, bad):
    """A row of V that is not finite, among the sinks, before the chunk and in it:
    tokens past its window are as without."""
    window, sinks = 64, 4
    print(f"[case] window leaves a row {at} {bad}", flush=True)
    p = Paged([150], [120], 2, 128, seed=7)
    p.rows[0][1][:, at] = bad
    p.write()
    q = queries(120, 4, 128, seed=1)
    ref, bound = reference(p, q, window_seen(p, window, sinks), out=F32)
    assert np.isfinite(ref).any() == (at > 3)
    check_close(_run(p, q, F32, window, sinks), ref, bound)


@pytest.mark.parametrize("sinks", [0, 7])
def test_a_window_that_hides_nothing(gpu_lib, sinks):
    print("[case] window hides nothing", flush=True)
    p = Paged([1500, 3, 260], [1, 300, 40], 2, 128, seed=8).write()
    q = queries(341, 8, 128, seed=8).cuda()
    plain, out = (torch.empty((341, 8, 128), dtype=BF16, device="cuda") for _ in range(2))
    ChunkAttention(p.cache, 8).run(p.chunks(), q, plain)
    ChunkAttention(p.cache, 8, window=1501, sinks=sinks).run(p.chunks(), q, out)
    torch.cuda.synchronize()
    assert torch.equal(plain, out)


def test_scale_strides_and_a_later_layer(gpu_lib):
    print("[case] window strides", flush=True)
    p = Paged([70, 400], [90, 5], 2, 64, layers=3, seed=4, gap=16).write()
    wide = torch.full((96, 10, 72), float("nan"), dtype=BF16, device="cuda")
    q = queries(95, 6, 64, seed=9)
    wide[:95, 2:8, :64] = q.cuda()
    out = torch.empty((95, 6, 64), dtype=F32, device="cuda")
    ChunkAttention(p.cache, 6, 0.3, window=40, sinks=3).run(p.chunks(), wide[:, 2:8, :64], out, layer=2)
    check_close(out, *reference(p, q, window_seen(p, 40, 3), layer=2, scale=0.3, out=F32))


def test_pages_past_4_gib(gpu_lib):
    row = 2 * 128 * 2
    spare = (1 << 32) // (64 * row) + 100
    print(f"[case] window pool of {spare * 64 * row / 2**30:.2f} GiB", flush=True)
    p = Paged([700, 900], [64, 1], 2, 128, spare=spare, far=True, seed=3).write()
    q = queries(65, 8, 128, seed=3)
    check_close(_run(p, q, F32, 300, 4), *reference(p, q, window_seen(p, 300, 4), out=F32))
    del p
    torch.cuda.empty_cache()


def test_captured_and_repeated(gpu_lib):
    """A captured call with a workspace and staging of its own, replayed beside
    eager calls of an object on other streams: the same bits."""
    print("[case] window replay", flush=True)
    p = Paged([1000, 3000, 10], [130, 1, 700], 2, 128, seed=12).write()
    q = queries(831, 8, 128, seed=12).cuda()
    att = ChunkAttention(p.cache, 8, window=600, sinks=4)
    first, out = (torch.empty((831, 8, 128), dtype=BF16, device="cuda") for _ in range(2))
    chunks, window = p.chunks(), B.SpecWindow(600, 4)
    att.run(chunks, q, first)
    a = B.SpecChunkAttnArgs()
    a.num_q_heads, a.out_dtype, a.q, a.out = 8, B.SPEC_BF16, q.data_ptr(), out.data_ptr()
    a.q_stride_tok, a.q_stride_head = 1024, 128
    st, dev, host = B.spec_chunk_window_workspace_bytes(chunks, p.cache.c, a, window)
    assert st == B.SPEC_OK
    ws = torch.empty(dev + 256, dtype=torch.uint8, device="cuda")
    staging = torch.empty(host, dtype=torch.uint8, pin_memory=True)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        B.check(B.spec_chunk_attn_window(chunks, p.cache.c, a, window, (ws.data_ptr() + 255) // 256 * 256, dev,
                                         staging.data_ptr(), host, stream.cuda_stream), "window")
        with pytest.raises(RuntimeError):
            att.run(chunks, q, out, stream=stream)
    other = torch.empty_like(first)
    for i in range(4):
        out.fill_(9.0)
        graph.replay()
        att.run(chunks, q, other, stream=None if i % 2 else stream)
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(other, first)
