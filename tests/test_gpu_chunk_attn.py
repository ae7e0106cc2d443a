"""GPU: attention of new tokens over a paged cache against its definition in
64 bits.  Every place of the pools that no request owns is NaN."""
import numpy as np
import pytest
import torch

from cache_util import BF16, F32, Paged, check_close, queries, reference
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention

pytestmark = pytest.mark.gpu

CASES = {
    # name: ctx, new, query heads, KV heads, d, page tokens
    "first_token": ([0], [1], 4, 4, 128, 32),
    "one_token_each": ([0, 1, 31, 32, 63, 64, 65, 700], [1] * 8, 8, 2, 128, 32),
    "decode_long": ([5000, 1023, 2048], [1, 1, 1], 8, 1, 128, 64),
    "few_tokens": ([100, 0, 37], [3, 8, 5], 8, 2, 64, 64),
    "prompt": ([0], [333], 8, 2, 128, 64),
    "prompt_mha": ([0, 0], [65, 128], 4, 4, 64, 96),
    "chunk_after_context": ([500, 77], [200, 129], 8, 2, 128, 96),
    "group_of_three": ([90, 10], [50, 43], 12, 4, 128, 32),
    "wide_group": ([300], [37], 40, 1, 64, 160),
    "with_nothing_new": ([40, 100, 7, 9], [0, 60, 0, 33], 8, 2, 128, 64),
    "mixed": ([1500, 3, 260, 0, 900], [1, 300, 1, 64, 31], 8, 2, 128, 64),
    "long_cut": ([6000], [40], 8, 2, 128, 256),
    "tile_edges": ([63, 64, 65, 127, 0], [65, 64, 63, 1, 32], 4, 1, 128, 32),
}


def _run(p, q, out_dtype, scale=0.0, layer=0):
    out = torch.full((q.shape[0] + 3, q.shape[1], q.shape[2]), 7.0, dtype=out_dtype, device="cuda")
    att = ChunkAttention(p.cache, q.shape[1], scale)
    att.run(p.chunks(), q.cuda(), out, layer=layer)
    torch.cuda.synchronize()
    assert (out[q.shape[0]:] == 7.0).all()               # rows past the last new token
    return out[:q.shape[0]]


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("name", CASES)
def test_matches_the_definition(gpu_lib, name, out):
    ctx, new, hq, hkv, d, page = CASES[name]
    print(f"[case] chunk {name} {out}", flush=True)
    p = Paged(ctx, new, hkv, d, page, seed=len(name)).write()
    q = queries(sum(new), hq, d, seed=len(name))
    check_close(_run(p, q, out), *reference(p, q, out=out))


@pytest.mark.parametrize("scale", [0.05, 3.0])
def test_scale_and_a_later_layer(gpu_lib, scale):
    print(f"[case] chunk scale {scale}", flush=True)
    p = Paged([70, 400], [90, 5], 2, 128, layers=3, seed=4).write()
    q = queries(95, 8, 128, seed=9)
    check_close(_run(p, q, F32, scale, layer=2), *reference(p, q, layer=2, scale=scale, out=F32))


@pytest.mark.parametrize("d", [64, 128])
def test_strided_queries_and_rows(gpu_lib, d):
    """Queries taken from a wider array, KV heads with a gap between them."""
    print(f"[case] chunk strides d {d}", flush=True)
    p = Paged([33, 150], [70, 1], 2, d, seed=2, gap=16).write()
    wide = torch.full((71, 10, d + 8), float("nan"), dtype=BF16, device="cuda")
    q = queries(71, 6, d, seed=3)
    wide[:, 2:8, :d] = q.cuda()
    out = torch.empty((71, 6, d), dtype=F32, device="cuda")
    ChunkAttention(p.cache, 6).run(p.chunks(), wide[:, 2:8, :d], out)
    check_close(out, *reference(p, q, out=F32))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", [6, 90])
def test_later_tokens_do_not_reach_earlier_ones(gpu_lib, bad, out, new):
    """A new token's K and V that are not finite: the tokens before it are as
    without, the ones from it on are not finite."""
    print(f"[case] chunk not finite {bad} {out} {new}", flush=True)
    p = Paged([50, 128], [new, 40], 2, 128, seed=6)
    at = 50 + new // 2
    kk, vv = p.rows[0]
    vv[:, at] = bad
    p.write()
    q = queries(new + 40, 4, 128, seed=1)
    ref, bound = reference(p, q, out=out)
    assert np.isfinite(ref[:new // 2]).all() and not np.isfinite(ref[new // 2:new]).any()
    check_close(_run(p, q, out), ref, bound)
    kk[:, at] = float("nan")
    p.write()
    got = _run(p, q, out)[:new // 2].double().cpu().numpy()
    assert (np.abs(got - ref[:new // 2]) <= bound[:new // 2]).all()


def test_large_scores(gpu_lib):
    """Scores of a few thousand: one key takes all the weight; the reference
    moves by more than any exponent in reach."""
    print("[case] chunk large scores", flush=True)
    p = Paged([300], [70], 1, 64, seed=8)
    kk, _ = p.rows[0]
    kk *= torch.linspace(1, 300, 370)[None, :, None, None].to(kk.dtype)
    p.write()
    q = queries(70, 2, 64, seed=2)
    got = _run(p, q, F32)
    ref, bound = reference(p, q, out=F32)
    check_close(got, ref, bound)


def test_pages_past_4_gib(gpu_lib):
    """A pool of over 4 GiB, the requests' pages at its end."""
    row = 2 * 128 * 2
    spare = (1 << 32) // (64 * row) + 100
    print(f"[case] chunk pool of {spare * 64 * row / 2**30:.2f} GiB", flush=True)
    p = Paged([700, 90], [64, 1], 2, 128, spare=spare, far=True, seed=3).write()
    q = queries(65, 8, 128, seed=3)
    check_close(_run(p, q, F32), *reference(p, q, out=F32))
    del p
    torch.cuda.empty_cache()


def test_same_bits_again_and_on_other_streams(gpu_lib):
    print("[case] chunk repeats", flush=True)
    p = Paged([1000, 3000, 10], [130, 1, 700], 2, 128, seed=12).write()
    q = queries(831, 8, 128, seed=12).cuda()
    att = ChunkAttention(p.cache, 8)
    first = torch.empty((831, 8, 128), dtype=BF16, device="cuda")
    att.run(p.chunks(), q, first)
    outs = [torch.empty_like(first) for _ in range(12)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):                          # one object, three streams in turn
        att.run(p.chunks(), q, o, stream=streams[i % 3])
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, first)


def test_pageable_staging(gpu_lib):
    """Staging that the device cannot map is copied ahead of the kernels."""
    print("[case] chunk pageable staging", flush=True)
    p = Paged([5000, 10], [60, 100], 2, 128, seed=14).write()
    q = queries(160, 8, 128, seed=14).cuda()
    ref = torch.empty((160, 8, 128), dtype=BF16, device="cuda")
    att = ChunkAttention(p.cache, 8)
    att.run(p.chunks(), q, ref)
    out = torch.empty_like(ref)
    att.args.out = out.data_ptr()
    st, dev, host = B.spec_chunk_workspace_bytes(p.chunks(), p.cache.c, att.args)
    B.check(st, "sizes")
    ws = torch.empty(dev + 256, dtype=torch.uint8, device="cuda")
    stage = np.zeros(host, np.uint8)
    ptr = (ws.data_ptr() + 255) // 256 * 256
    B.check(B.spec_chunk_attn(p.chunks(), p.cache.c, att.args, ptr, dev, stage.ctypes.data, host,
                              torch.cuda.current_stream().cuda_stream), "spec_chunk_attn")
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


def test_captured_and_replayed(gpu_lib):
    """Two captured calls with a workspace and staging of their own, replayed in
    turn between eager calls."""
    print("[case] chunk graphs", flush=True)
    stream = torch.cuda.Stream()
    made = []
    for k, (ctx, new) in enumerate([([4000, 30], [1, 1]), ([900, 0], [70, 200])]):
        p = Paged(ctx, new, 2, 128, seed=20 + k).write()
        q = queries(sum(new), 8, 128, seed=20 + k).cuda()
        ref, out = (torch.empty((sum(new), 8, 128), dtype=BF16, device="cuda") for _ in range(2))
        att = ChunkAttention(p.cache, 8)
        att.run(p.chunks(), q, ref)
        att.args.out = out.data_ptr()
        st, dev, host = B.spec_chunk_workspace_bytes(p.chunks(), p.cache.c, att.args)
        ws = torch.empty(dev + 256, dtype=torch.uint8, device="cuda")
        stage = torch.empty(host, dtype=torch.uint8, pin_memory=True)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            st = B.spec_chunk_attn(p.chunks(), p.cache.c, att.args, (ws.data_ptr() + 255) // 256 * 256, dev,
                                   stage.data_ptr(), host, torch.cuda.current_stream().cuda_stream)
        B.check(st, "captured")
        made.append((g, out, ref, att, p, q, ws, stage))
    for rep in range(4):
        for g, out, ref, att, p, q, *_ in made:
            out.zero_()
            g.replay()
            again = torch.empty_like(ref)
            att.run(p.chunks(), q, again)
            torch.cuda.synchronize()
            assert torch.equal(out, ref) and torch.equal(again, ref), rep


def test_page_ids_outside_the_pool(gpu_lib):
    """Page ids outside [0, num_pages) are clamped into the pool: that request's
    rows mean nothing, the others' are as before."""
    print("[case] chunk page ids outside", flush=True)
    p = Paged([200, 300], [40, 50], 2, 128, seed=5, fill=0.0).write()
    q = queries(90, 8, 128, seed=5)
    good = _run(p, q, BF16)
    p.table[0, 1], p.table[0, 2] = -5, 1 << 30
    got = _run(p, q, BF16)
    assert torch.equal(got[40:], good[40:])


def _device_case(B_, n, ctx, hkv, G, d, page, seed):
    """Large pools made on the device; returns (cache, table, ctx, q)."""
    from paper_2505_17074_amd.cache import PagedCache
    g = torch.Generator(device="cuda").manual_seed(seed)
    per = -(-(ctx + n) // page)
    order = torch.randperm(B_ * per + 2, generator=g, device="cuda")[:B_ * per].to(torch.int32).view(B_, per)
    k, v = (torch.randn((1, B_ * per + 2, page, hkv, d), generator=g, device="cuda", dtype=BF16) for _ in range(2))
    q = torch.randn((B_ * n, hkv * G, d), generator=g, device="cuda", dtype=BF16)
    return PagedCache(k, v, order.contiguous()), q


@pytest.mark.parametrize("B_,n,ctx,hkv,G,d", [(43, 1, 2111, 32, 1, 64), (64, 32, 2500, 8, 4, 128)],
                         ids=["one_wave", "four_waves"])
def test_items_of_more_than_2048_keys(gpu_lib, B_, n, ctx, hkv, G, d):
    """Batches whose items are not cut at all: the page ids of an item come in
    several windows.  A few requests against the definition, on the device."""
    print(f"[case] chunk long items {B_} {n} {ctx}", flush=True)
    cache, q = _device_case(B_, n, ctx, hkv, G, d, 96, 5)
    out = torch.empty((B_ * n, hkv * G, d), dtype=F32, device="cuda")
    ChunkAttention(cache, hkv * G).run(B.make_chunks([ctx] * B_, [n] * B_), q, out)
    seen = torch.arange(ctx + n, device="cuda")[None] <= ctx + torch.arange(n, device="cuda")[:, None]
    for i in (0, B_ // 2, B_ - 1):
        kk, vv = (x[0, cache.table[i].long()].reshape(-1, hkv, d)[:ctx + n].double() for x in (cache.k, cache.v))
        for h in range(hkv * G):
            qq = q[i * n:(i + 1) * n, h].double()
            s = torch.where(seen, (qq @ kk[:, h // G].t().contiguous()) / d ** 0.5, -float("inf"))
            w = torch.softmax(s, -1)
            ref, size = w @ vv[:, h // G], w @ vv[:, h // G].abs()
            e = (d + 6) * 2.0 ** -24 * 1.4427 * float(qq.abs().max() * kk.abs().max()) * d ** 0.5
            bound = size * (2 * e + 2.0 ** -24 + (2 * (ctx + n) + 16) * 2.0 ** -24) + 2.0 ** -24 * ref.abs()
            assert ((out[i * n:(i + 1) * n, h].double() - ref).abs() <= bound * 1.01).all(), (i, h)


def test_keys_and_values_in_one_tensor(gpu_lib):
    """K and V interleaved by token: views of one [.., 2, Hkv, d] allocation."""
    from paper_2505_17074_amd.cache import PagedCache
    print("[case] chunk interleaved", flush=True)
    p = Paged([200, 40], [60, 1], 2, 64, 32, layers=2, seed=9).write()
    both = torch.full((2, p.num_pages, 32, 2, 2, 64), float("nan"), dtype=BF16, device="cuda")
    both[:, :, :, 0], both[:, :, :, 1] = p.k, p.v
    cache = PagedCache(both[:, :, :, 0], both[:, :, :, 1], p.table)
    q = queries(61, 8, 64, seed=9)
    out = torch.empty((61, 8, 64), dtype=F32, device="cuda")
    ChunkAttention(cache, 8).run(p.chunks(), q.cuda(), out, layer=1)
    check_close(out, *reference(p, q, layer=1, out=F32))
    k_new, v_new = (torch.randn((2, 61, 2, 64)).to(BF16).cuda() for _ in range(2))
    cache.append(p.chunks(), k_new, v_new)
    torch.cuda.synchronize()
    q0 = 0
    for i in range(2):
        c, n = int(p.ctx[i]), int(p.new[i])
        pg, pl = (torch.from_numpy(x).cuda() for x in p.where(i, np.arange(c, c + n)))
        assert torch.equal(both[:, pg, pl, 0], k_new[:, q0:q0 + n]) and torch.equal(both[:, pg, pl, 1], v_new[:, q0:q0 + n])
        q0 += n


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(gpu_lib, seed):
    rng = np.random.default_rng(100 + seed)
    b = int(rng.integers(1, 7))
    ctx = [int(x) for x in rng.integers(0, rng.choice([3, 70, 600]), b)]
    new = [int(x) for x in rng.integers(0, rng.choice([2, 9, 150]), b)]
    new[0] = max(new[0], 1)
    hkv, G = int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 4, 5, 8]))
    d, page, out = int(rng.choice([64, 128])), int(rng.choice([32, 64, 96, 256])), [BF16, F32][seed % 2]
    print(f"[case] chunk random {seed} ctx {ctx} new {new} heads {hkv * G}/{hkv} d {d} page {page}", flush=True)
    p = Paged(ctx, new, hkv, d, page, seed=seed, layers=1 + seed % 2).write()
    q = queries(sum(new), hkv * G, d, seed=seed)
    check_close(_run(p, q, out, layer=seed % 2), *reference(p, q, layer=seed % 2, out=out))


def test_one_object_for_growing_batches(gpu_lib):
    """Workspace and staging grow with the batches; a large one between small
    ones, back to back."""
    print("[case] chunk growing", flush=True)
    p = Paged([900, 3000, 5, 77], [1, 1, 130, 64], 2, 128, seed=30).write()
    att = ChunkAttention(p.cache, 8)
    table = p.table.clone()
    want, outs = [], []
    for sel in ([0], [2, 3], [0, 1, 2, 3], [0], [1], [0, 1, 2, 3]):
        q = queries(int(p.new[sel].sum()), 8, 128, seed=len(sel))
        out = torch.empty((q.shape[0], 8, 128), dtype=BF16, device="cuda")
        p.cache.table = table[sel].contiguous()
        outs.append((p.cache.table, q.cuda(), out))
        att.run(B.make_chunks(p.ctx[sel], p.new[sel]), outs[-1][1], out)
        sub = Paged.__new__(Paged)
        sub.ctx, sub.new, sub.hkv, sub.rows = p.ctx[sel], p.new[sel], 2, [p.rows[i] for i in sel]
        want.append(reference(sub, q))
    for (_, _, out), (ref, bound) in zip(outs, want):
        check_close(out, ref, bound)


def test_objects_that_end_with_work_pending(gpu_lib):
    """Staging and workspace stay until the call that uses them has ended,
    whoever takes their memory next."""
    print("[case] chunk objects ending early", flush=True)
    p = Paged([900, 3000, 5, 77], [1, 1, 130, 64], 2, 128, seed=31).write()
    q = queries(196, 8, 128, seed=31).cuda()
    ref, out = (torch.empty((196, 8, 128), dtype=BF16, device="cuda") for _ in range(2))
    ChunkAttention(p.cache, 8).run(p.chunks(), q, ref)
    side = torch.cuda.Stream()
    a = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(4):
        out.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(8):
                torch.mm(a, a)                            # the call below waits behind these
        att = ChunkAttention(p.cache, 8)
        att.run(p.chunks(), q, out, stream=side)
        sizes = att._pinned.numel(), att._ws.numel()
        del att
        torch.empty(sizes[0], dtype=torch.uint8, pin_memory=True).fill_(0)
        torch.empty(sizes[1], dtype=torch.uint8, device="cuda").fill_(255)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


FEW = [0, 1, 30, 31, 32, 33, 62, 63, 64, 65, 127, 128, 129, 191, 700, 2047, 4200]


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new,hkv,G", [(1, 2, 4), (1, 1, 1), (8, 2, 4), (5, 2, 3), (32, 1, 1)])
def test_few_rows_beside_many(gpu_lib, new, hkv, G, out):
    """Requests of up to 32 query rows a KV head in a batch with a longer one."""
    print(f"[case] chunk few beside many {new} {hkv} {G} {out}", flush=True)
    p = Paged(FEW + [90], [new] * len(FEW) + [150], hkv, 128, 32, seed=new + G).write()
    q = queries(new * len(FEW) + 150, hkv * G, 128, seed=G)
    check_close(_run(p, q, out), *reference(p, q, out=out))


def test_few_rows_cut_beside_many(gpu_lib):
    """A request of few rows whose keys are cut into pieces."""
    print("[case] chunk few rows cut", flush=True)
    p = Paged([9000, 10], [2, 80], 1, 128, 64, seed=77).write()
    q = queries(82, 4, 128, seed=5)
    check_close(_run(p, q, F32), *reference(p, q, out=F32))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [40, 52, 54, 100, 133])
def test_few_rows_beside_many_not_finite(gpu_lib, at, bad):
    """A V row that is not finite, by where it falls among the waves' shares:
    seen by all tokens of the first request, by some, and by none of the second's."""
    print(f"[case] chunk few rows not finite {at} {bad}", flush=True)
    p = Paged([50, 128, 3], [6, 7, 70], 2, 128, seed=16)
    i = 0 if at < 56 else 1
    p.rows[i][1][:, at] = bad
    p.write()
    q = queries(83, 8, 128, seed=1)
    ref, bound = reference(p, q, out=F32)
    assert not np.isfinite(ref).all() and np.isfinite(ref[13:]).all()
    check_close(_run(p, q, F32), ref, bound)
