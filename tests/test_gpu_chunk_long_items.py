"""GPU: requests of few query rows beside longer ones (all four waves share
their keys), over key ranges that are not cut: past the first window of page ids
(2048 keys) and through many turns of the ring."""
import pytest
import torch

from cache_util import BF16, F32, U32
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention, PagedCache

pytestmark = pytest.mark.gpu

D, P = 128, 32
BATCHES = {
    # name: KV heads, heads a group, few-row requests (cached rows, new tokens), longer ones
    "single_tokens": (32, 1, [(2100, 1), (2047, 1), (3003, 1), (4500, 1), (64, 1)], [(1500, 400)] * 6),
    "groups": (8, 4, [(2300, 8), (4100, 3), (2049, 7), (31, 1)], [(1700, 512)] * 5),
}


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [False, True], ids=["finite", "not_finite"])
@pytest.mark.parametrize("name", BATCHES)
def test_few_rows_over_long_whole_items(gpu_lib, name, bad, out):
    hkv, G, few, more = BATCHES[name]
    print(f"[case] chunk long few-row items {name} {bad} {out}", flush=True)
    # the longer ones between the others, so that neither kind stands together
    reqs = [r for pair in zip(few, more) for r in pair] + more[len(few):] + few[len(more):]
    ctx, new = [r[0] for r in reqs], [r[1] for r in reqs]
    pages = [-(-(c + n) // P) for c, n in reqs]
    g = torch.Generator(device="cuda").manual_seed(len(name))
    order = torch.randperm(sum(pages) + 3, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(reqs), max(pages)), 1 << 30, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = order[at:at + n]
        at += n
    k, v = (torch.randn((1, sum(pages) + 3, P, hkv, D), generator=g, device="cuda", dtype=BF16) for _ in range(2))
    q = torch.randn((sum(new), hkv * G, D), generator=g, device="cuda", dtype=BF16)
    spoiled = {}
    if bad:                                              # one element of V each, past key 2048 where there are so many
        for i, (c, n) in enumerate(reqs):
            if n <= 8 and c > 2048:
                t, col = (2048 + c) // 2, 3 + i
                v[0, table[i, t // P].long(), t % P, i % hkv, col] = [float("nan"), float("inf")][i % 2]
                spoiled[i] = (i % hkv, col)
    cache, chunks = PagedCache(k, v, table), B.make_chunks(ctx, new)
    got = torch.empty((sum(new), hkv * G, D), dtype=out, device="cuda")
    att = ChunkAttention(cache, hkv * G)
    att.run(chunks, q, got)
    # no partial rows: no item of this batch is cut, whatever the rule is then
    att.args.out_dtype = B.SPEC_BF16 if out == BF16 else B.SPEC_F32
    st, dev, host = B.spec_chunk_workspace_bytes(chunks, cache.c, att.args)
    assert st == B.SPEC_OK and dev == host, "the batch is cut: it no longer tests what it is for"
    p_part, rounding = (2.0 ** -8, 2.0 ** -8) if out == BF16 else (U32, U32)
    q0 = 0
    for i, (c, n) in enumerate(reqs):
        rows = slice(q0, q0 + n)
        q0 += n
        if n > 8 and i != 1:
            continue                                     # of the longer ones, one
        kk, vv = (x[0, table[i, :pages[i]].long()].reshape(-1, hkv, D)[:c + n].double() for x in (k, v))
        seen = torch.arange(c + n, device="cuda")[None] <= c + torch.arange(n, device="cuda")[:, None]
        for h in range(hkv * G):
            qq, kh, vh = q[rows, h].double(), kk[:, h // G], vv[:, h // G]
            s = torch.where(seen, torch.mm(qq, kh.t().contiguous()) / D ** 0.5, -float("inf"))
            w = torch.softmax(s, -1)
            v0 = torch.nan_to_num(vh, 0.0, 0.0, 0.0)
            ref, size = torch.mm(w, v0), torch.mm(w, v0.abs())
            # fp32 dot products of 128 terms, the scale and the subtraction: an error of the exponent
            e = (D + 6) * U32 * 1.4427 * float(qq.abs().max() * kh.abs().max()) * D ** 0.5
            bound = size * (p_part + 2 * e + (2 * (c + n) + 16) * U32) + rounding * ref.abs()
            y = got[rows, h].double()
            fine = torch.ones(D, dtype=torch.bool, device="cuda")
            if i in spoiled and spoiled[i][0] == h // G:
                fine[spoiled[i][1]] = False
                assert not torch.isfinite(y[:, ~fine]).any(), (i, h)
            assert ((y - ref).abs() <= bound * 1.01)[:, fine].all(), (i, h)
