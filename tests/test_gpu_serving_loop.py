"""GPU: the operators around the verify step as one loop uses them: a prompt
appended with the rotation, attention in windows and over everything, forks that
share the prompt, sampled tokens that become the next rows."""
import numpy as np
import pytest
import torch

import oracle
from attend_util import reference, window_seen
from cache_util import BF16, F32, check_close
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention, PagedCache, Pages
from paper_2505_17074_amd.sample import Sampler
from test_gpu_rotate import _check as check_turned, _freq, turned

pytestmark = pytest.mark.gpu

HQ, HKV, D, P, V = 8, 2, 128, 32, 700
WINDOW, SINKS = 50, 4


class Rows:
    """What attend_util.reference reads: the requests' rows as the cache holds them."""

    def __init__(self, cache, tables, ctx, new):
        self.ctx, self.new, self.hkv = np.asarray(ctx), np.asarray(new), HKV
        self.rows = []
        for table, c, n in zip(tables, ctx, new):
            t = np.arange(c + n)
            page, place = torch.from_numpy(table[t // P].astype(np.int64)).cuda(), torch.from_numpy(t % P).cuda()
            self.rows.append(tuple(x[:, page, place].cpu() for x in (cache.k, cache.v)))


def test_a_serving_loop(gpu_lib):
    print("[case] serving loop", flush=True)
    g = torch.Generator().manual_seed(1)
    embed = {x: torch.randn((V, h, D), generator=g).to(BF16).cuda() for x, h in (("q", HQ), ("k", HKV), ("v", HKV))}
    head = (torch.randn((HQ * D, V), generator=g) * 0.3).cuda()
    k = torch.full((1, 60, P, HKV, D), float("nan"), dtype=BF16, device="cuda")
    cache, pages = PagedCache(k, k.clone()), Pages(60, P)
    whole, windowed, sampler = ChunkAttention(cache, HQ), ChunkAttention(cache, HQ, window=WINDOW, sinks=SINKS), Sampler()
    freq = _freq(D).cuda()

    def step(sequences, ctx, tokens, prefixes=None):
        """The tokens' rows behind each sequence's ctx; their outputs, in windows and over everything."""
        new = [len(t) for t in tokens]
        for s, c, n in zip(sequences, ctx, new):
            copy = pages.resize(s, c + n)
            if copy:
                cache.copy_pages([copy])
        cache.table = torch.from_numpy(pages.block_table(sequences)).cuda()
        ids = torch.tensor([x for t in tokens for x in t], device="cuda")
        chunks = B.make_chunks(ctx, new)
        q, kk, vv = (embed[x][ids].contiguous() for x in ("q", "k", "v"))
        turned_q = torch.empty_like(q)
        cache.append_rotated(chunks, kk, vv, freq, q, turned_q)
        near, out = torch.empty((len(ids), HQ, D), dtype=BF16, device="cuda"), torch.empty((len(ids), HQ, D), dtype=F32, device="cuda")
        windowed.run(chunks, turned_q, near)
        whole.run(chunks, turned_q, out, prefixes=prefixes)
        torch.cuda.synchronize()
        tables = [pages.table(s) for s in sequences]
        rows = Rows(cache, tables, ctx, new)
        at = np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, new)])
        check_turned(turned_q, *turned(q, at, freq.cpu(), False, BF16))
        mine = torch.cat([r[0][0, c:] for r, c in zip(rows.rows, ctx)])
        check_turned(mine, *turned(kk, at, freq.cpu(), False, BF16))
        assert torch.equal(torch.cat([r[1][0, c:] for r, c in zip(rows.rows, ctx)]), vv.cpu())
        check_close(near, *reference(rows, turned_q.cpu(), window_seen(rows, WINDOW, SINKS)))
        check_close(out, *reference(rows, turned_q.cpu(), window_seen(rows, 1 << 40, 0), out=F32))
        return out

    def draw(out, seed):
        """A token of each row."""
        logits = out.reshape(out.shape[0], -1) @ head
        n = logits.shape[0]
        u = torch.rand(n, generator=torch.Generator().manual_seed(seed)).cuda()
        T, top_k, top_p = torch.full((n,), 0.9, device="cuda"), torch.full((n,), 40, dtype=torch.int32, device="cuda"), \
            torch.full((n,), 0.95, device="cuda")
        tokens, probs = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty_like(logits)
        sampler.run(logits, u, tokens, temperature=T, top_k=top_k, top_p=top_p, probs=probs)
        x = logits.double().cpu().numpy()
        for i in range(n):
            token, want, _, margin = oracle.sample(x[i], u[i].item(), T[i].item(), 40, top_p[i].item())
            if margin > 4e-10:
                assert tokens[i].item() == token
                assert (np.abs(probs[i].double().cpu().numpy() - want) <= want * 2.0 ** -23 + 2.0 ** -126).all()
        return tokens.tolist()

    prompt = torch.randint(0, V, (300,), generator=g).tolist()
    s = pages.open()
    step([s], [0], [prompt[:150]])
    out = step([s], [150], [prompt[150:]])
    first = draw(out[-1:].expand(3, HQ, D).contiguous(), 7)                 # three answers
    family = [s, pages.fork(s), pages.fork(s)]
    own = [[t] for t in first]
    for i in range(4):
        ctx = [300 + len(t) - 1 for t in own]
        out = step(family, ctx, [t[-1:] for t in own], B.make_prefixes([3], [300]))
        for t, x in zip(own, draw(out, 20 + i)):
            t.append(x)
    assert pages.free == 60 - (300 // P) - 3                               # the prompt's whole pages are shared
    for x in family:
        pages.close(x)
    assert pages.free == 60
