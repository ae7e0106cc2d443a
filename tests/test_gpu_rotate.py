"""GPU: appended rows with the position rotation against its definition in 64
bits.  The pools are NaN wherever no row was written."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from cache_util import BF16, F32, Paged, queries
from paper_2505_17074_amd import binding as B

pytestmark = pytest.mark.gpu

CASES = {
    # name: ctx, new, query heads, KV heads, d, page tokens, rotated elements
    "first_token": ([0], [1], 4, 4, 128, 32, 128),
    "one_token_each": ([0, 1, 31, 32, 63, 700], [1] * 6, 8, 2, 128, 32, 128),
    "half_of_a_head": ([3, 500], [9, 2], 8, 2, 128, 64, 64),
    "small_heads": ([100, 0, 37], [3, 8, 5], 8, 2, 64, 64, 64),
    "prompt": ([7], [333], 8, 2, 128, 96, 128),
    "nothing_new": ([40, 100, 7], [0, 60, 0], 12, 4, 128, 64, 32),
    "odd_heads": ([40, 100], [31, 33], 5, 3, 96, 32, 96),
    "one_head": ([9], [66], 1, 1, 32, 32, 16),
    "wide_heads": ([5, 60], [3, 6], 3, 2, 576, 32, 512),
    "many_requests": (list(range(300)), [1 + i % 3 for i in range(300)], 4, 2, 64, 32, 64),
}


def _freq(rotary, base=10000.0):
    return torch.tensor([base ** (-2 * i / rotary) for i in range(rotary // 2)], dtype=torch.float32)


def turned(x, pos, freq, interleaved, dtype):
    """x [rows, heads, d] turned in 64 bits, and a bound on the kernel's distance:
    cos and sin off by 2^-23, two products and a sum in fp32, half a step."""
    x = x.double().cpu().numpy()
    a = pos.astype(np.float64)[:, None] * freq.double().numpy()[None]
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    half = freq.shape[0]
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y, size = x.copy(), np.zeros_like(x)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    size[..., i] = size[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    half_step = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    return y, size * (2.0 ** -23 + 2.0 ** -23) * (1 + half_step) + half_step * np.abs(y) * (size > 0)


def _check(got, ref, bound):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bound * 1.01 + 1e-38).all(), float((np.abs(got - ref) - bound).max())


def _rows(p):
    """The new rows as they lie in the pools [Nq, Hkv, d], K and V; everything else is NaN."""
    out = []
    for pool in (p.k, p.v):
        rows, seen = [], torch.zeros(pool.shape[1:3], dtype=torch.bool)
        for i in range(len(p.new)):
            pg, pl = p.where(i, np.arange(p.ctx[i], p.ctx[i] + p.new[i]))
            rows.append(pool[0, torch.from_numpy(pg).cuda(), torch.from_numpy(pl).cuda()])
            seen[torch.from_numpy(pg), torch.from_numpy(pl)] = True
        assert torch.isnan(pool[0][~seen.cuda()]).all()
        out.append(torch.cat(rows))
    return out


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("name", CASES)
def test_matches_the_definition(gpu_lib, name, dtype, interleaved):
    ctx, new, hq, hkv, d, page, rotary = CASES[name]
    print(f"[case] rotate {name} {dtype} {interleaved}", flush=True)
    p = Paged(ctx, new, hkv, d, page, dtype=dtype, seed=len(name))
    k, v = (x[0] for x in p.new_rows())
    n = sum(new)
    q = queries(n + 2, hq, d, seed=len(name), dtype=dtype).cuda()
    q_out = torch.full_like(q, 7.0)
    freq = _freq(rotary)
    before = k.clone(), v.clone(), q.clone()
    p.cache.append_rotated(p.chunks(), k, v, freq.cuda(), q, q_out, interleaved=interleaved)
    torch.cuda.synchronize()
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(ctx, new)])
    assert (q_out[n:] == 7.0).all()
    assert all(torch.equal(x, y) for x, y in zip(before, (k, v, q)))
    _check(q_out[:n], *turned(q[:n], pos, freq, interleaved, dtype))
    kk, vv = _rows(p)
    _check(kk, *turned(k, pos, freq, interleaved, dtype))
    assert torch.equal(vv, v)


def test_far_and_given_positions(gpu_lib):
    """Positions of up to 2^31 radians and below zero, in place, without a
    queries' head gap and with one."""
    print("[case] rotate positions", flush=True)
    pos = np.array([0, 1, -1, 12345, 1 << 20, (1 << 24) + 1, 2**31 - 1, -2**31, 99999999], np.int32)
    p = Paged([50, 3], [5, 4], 2, 128, seed=1, dtype=F32, gap=16)
    k, v = (x[0] for x in p.new_rows())
    wide = torch.zeros((9, 6, 160), dtype=F32, device="cuda")
    q = wide[:, 1:5, :128]
    q.copy_(queries(9, 4, 128, seed=1, dtype=F32))
    was = q.clone()
    freq = _freq(128, 500000.0)
    p.cache.append_rotated(p.chunks(), k, v, freq.cuda(), q, q, positions=torch.from_numpy(pos).cuda())
    torch.cuda.synchronize()
    _check(q, *turned(was, pos, freq, False, F32))
    _check(_rows(p)[0], *turned(k, pos, freq, False, F32))
    assert (wide[:, 0] == 0).all() and (wide[:, 5] == 0).all() and (wide[..., 128:] == 0).all()


def test_layers_without_queries(gpu_lib):
    print("[case] rotate layers", flush=True)
    p = Paged([40, 0, 99], [7, 70, 1], 2, 64, layers=3, seed=2)
    k, v = p.new_rows()
    freq = _freq(64)
    p.cache.append_rotated(p.chunks(), k[1:], v[1:], freq.cuda(), layer=1)
    torch.cuda.synchronize()
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(p.ctx, p.new)])
    assert torch.isnan(p.k[0]).all() and torch.isnan(p.v[0]).all()
    for layer in (1, 2):
        one = Paged([40, 0, 99], [7, 70, 1], 2, 64, seed=2)
        one.k, one.v = p.k[layer:layer + 1], p.v[layer:layer + 1]
        kk, vv = _rows(one)
        _check(kk, *turned(k[layer], pos, freq, False, BF16))
        assert torch.equal(vv, v[layer])


def test_turned_back(gpu_lib):
    """Scores depend on the distance alone: q at position t + a with k at t
    gives the same product for every t, within fp32."""
    print("[case] rotate distances", flush=True)
    n = 64
    p = Paged([0], [n], 1, 64, dtype=F32, seed=3)
    k = torch.randn((1, 1, 64), device="cuda").expand(n, 1, 64).contiguous()
    q = torch.randn((1, 1, 64), device="cuda").expand(n, 1, 64).contiguous()
    pos = (torch.arange(n, device="cuda", dtype=torch.int32) * 12347)
    q_out = torch.empty_like(q)
    p.cache.append_rotated(p.chunks(), k, k, _freq(64).cuda(), q, q_out, positions=pos)
    s = (q_out.double() * _rows(p)[0].double()).sum(-1)[:, 0].cpu()
    size = (q[0].double().abs() * k[0].double().abs()).sum().item() * 2
    assert (s - s[0]).abs().max() <= size * 8 * 2.0 ** -23


def test_a_round_of_trees(gpu_lib):
    """Nodes rotated by ctx + depth: after the commit the accepted path's rows
    are what a chain of the same tokens would have put there."""
    print("[case] rotate tree", flush=True)
    par = np.array([-1, 0, 0, 1, 1, 2], np.int32)
    depth = np.array([0, 1, 1, 2, 2, 2], np.int32)
    path = [0, 2, 5]
    p = Paged([61, 10], [6, 6], 2, 128, seed=4)
    k, v = (x[0] for x in p.new_rows())
    freq = _freq(128).cuda()
    pos = torch.from_numpy(np.concatenate([61 + depth, 10 + depth]).astype(np.int32)).cuda()
    p.cache.append_rotated(p.chunks(), k, v, freq, positions=pos)
    p.cache.commit(B.make_requests([61, 10], None, par), torch.tensor([5, 5], dtype=torch.int32, device="cuda"))
    one = Paged([61, 10], [3, 3], 2, 128, seed=4)
    pick = path + [6 + x for x in path]
    one.cache.append_rotated(one.chunks(), k[pick], v[pick], freq)
    torch.cuda.synchronize()
    for i, c in enumerate((61, 10)):
        pg, pl = (torch.from_numpy(x).cuda() for x in p.where(i, np.arange(c, c + 3)))
        og, ol = (torch.from_numpy(x).cuda() for x in one.where(i, np.arange(c, c + 3)))
        assert torch.equal(p.k[0, pg, pl], one.k[0, og, ol]) and torch.equal(p.v[0, pg, pl], one.v[0, og, ol])


def test_pages_outside_the_pool_are_not_written(gpu_lib):
    print("[case] rotate bad pages", flush=True)
    p = Paged([0, 64], [40, 40], 2, 64, page=32, seed=5)
    k, v = (x[0] for x in p.new_rows())
    bad = p.table.clone()
    bad[0, 1], bad[1, 2] = p.num_pages, -1
    p.cache.table = bad
    q = queries(80, 4, 64).cuda()
    q_out = torch.zeros_like(q)
    p.cache.append_rotated(p.chunks(), k, v, _freq(64).cuda(), q, q_out)
    torch.cuda.synchronize()
    written = (~torch.isnan(p.k[0, :, :, 0, 0])).sum().item()
    assert written == 32 + 8
    assert (q_out != 0).any(-1).all()


def test_replayed_with_new_values(gpu_lib):
    """A captured call reads its tensors again at every replay."""
    print("[case] rotate replay", flush=True)
    p = Paged([33, 5], [4, 30], 2, 128, seed=6)
    k, v = (x[0] for x in p.new_rows())
    q, freq = queries(34, 8, 128).cuda(), _freq(128).cuda()
    q_out, pos = torch.empty_like(q), torch.arange(34, dtype=torch.int32, device="cuda")
    chunks = p.chunks()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        p.cache.append_rotated(chunks, k, v, freq, q, q_out, positions=pos, stream=stream)
    for i in range(3):
        pos.copy_(torch.randint(0, 100000, (34,), device="cuda", dtype=torch.int32))
        q.copy_(queries(34, 8, 128, seed=i))
        graph.replay()
        torch.cuda.synchronize()
        got_q, got_k = q_out.clone(), _rows(p)[0].clone()
        p.cache.append_rotated(chunks, k, v, freq, q, q_out, positions=pos)
        torch.cuda.synchronize()
        assert torch.equal(got_q, q_out) and torch.equal(got_k, _rows(p)[0])


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_heads_behind_each_other(gpu_lib, dtype, interleaved):
    """Queries [Hq, rows, d] seen as [rows, Hq, d], into another tensor of that
    order or of the usual one, and in place: the same values."""
    print(f"[case] rotate heads first {dtype} {interleaved}", flush=True)
    n, hq, d = 41, 6, 128
    p = Paged([30, 0], [38, 3], 2, d, seed=7, dtype=dtype)
    k, v = (x[0] for x in p.new_rows())
    q = queries(n, hq, d, seed=7, dtype=dtype).cuda()
    freq = _freq(d).cuda()
    want = torch.empty_like(q)
    p.cache.append_rotated(p.chunks(), k, v, freq, q, want, interleaved=interleaved)
    heads = torch.full((hq, n + 1, d + 16), 7.0, dtype=dtype, device="cuda")          # gaps between rows and heads
    view = heads[:, :n, :d].transpose(0, 1)
    p.cache.append_rotated(p.chunks(), k, v, freq, q, view, interleaved=interleaved)
    torch.cuda.synchronize()
    assert torch.equal(view, want) and (heads[:, n:] == 7.0).all() and (heads[..., d:] == 7.0).all()
    view.copy_(q)
    back = torch.empty_like(q)
    p.cache.append_rotated(p.chunks(), k, v, freq, view, back, interleaved=interleaved)
    p.cache.append_rotated(p.chunks(), k, v, freq, view, view, interleaved=interleaved)
    torch.cuda.synchronize()
    assert torch.equal(back, want) and torch.equal(view, want)
    assert (heads[:, n:] == 7.0).all() and (heads[..., d:] == 7.0).all()


PI = Fraction(31415926535897932384626433832795028841971693993751058209749445923, 10**64)     # 2^-212 off


def _cos_sin(p, f):
    """Of the exact product of a whole number and an fp32 number, to 2^-52 (the
    product's turns are taken off in fractions: 2^46 of them are off by 2^-160)."""
    a = Fraction(int(p)) * Fraction(float(f))
    r = float(a - round(a / (2 * PI)) * 2 * PI)
    return math.cos(r), math.sin(r)


@pytest.mark.parametrize("largest", [1.0, 8.0, 1000.0, 16384.0])
def test_cos_and_sin_of_any_angle(gpu_lib, largest):
    """Rows of (1, 0) pairs turn into the angles' cos and sin themselves: off by
    2^-23 at most, at all positions and frequencies up to 2^14."""
    print(f"[case] rotate angles up to {largest}", flush=True)
    rng = np.random.default_rng(int(largest))
    n, pairs = 256, 64
    pos = np.concatenate([rng.integers(-2**31, 2**31, 100), 2**31 - 1 - rng.integers(0, 1000, 50),
                          -2**31 + rng.integers(0, 1000, 20), rng.integers(-2**24, 2**24, 50), np.arange(-18, 18)])
    freq = (rng.random(pairs) * largest).astype(np.float32)
    freq[:3] = largest, -largest, np.nextafter(np.float32(largest), np.float32(0))
    p = Paged([0], [n], 1, 2 * pairs, dtype=F32, seed=8)
    k = torch.zeros((n, 1, 2 * pairs), dtype=F32, device="cuda")
    k[..., :pairs] = 1.0
    p.cache.append_rotated(p.chunks(), k, k, torch.from_numpy(freq).cuda(),
                           positions=torch.from_numpy(pos.astype(np.int32)).cuda())
    torch.cuda.synchronize()
    got = _rows(p)[0][:, 0].double().cpu().numpy()
    want = np.array([[_cos_sin(x, f) for f in freq] for x in pos]).transpose(0, 2, 1).reshape(n, 2 * pairs)
    assert np.abs(got - want).max() <= 2.0 ** -23, float(np.abs(got - want).max() * 2.0 ** 23)
