"""GPU: the paged cache's operators together, as a serving loop uses them.
Prompts come in chunks (resize, copies, append, attention), one request is
forked, and rounds of token trees follow (append, verify attention on the same
pools, acceptance, commit, resize).  A host model holds each request's rows;
every attention is compared with the definition on them in 64 bits, and every
accepted path is where the next round reads it."""

import numpy as np
import pytest
import torch

from cache_util import BF16, F32, U32, queries
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention, PagedCache, Pages

pytestmark = pytest.mark.gpu

HQ, HKV, D, P, LAYERS, VOCAB = 8, 2, 128, 32, 2, 500


def _attend(q, k, v, seen):
    """fp64 attention [n, HQ, D] of q over rows k, v [t, HKV, D] and its bound
    (bf16 weights: 2^-8 of the weights' sum; fp32 sums of d and t terms)."""
    n, G = q.shape[0], HQ // HKV
    q, k, v = (x.double().cpu().numpy() for x in (q, k, v))
    out, size = np.zeros((n, HQ, D)), np.zeros((n, HQ, D))
    for h in range(HQ):
        s = np.where(seen, q[:, h] @ k[:, h // G].T / np.sqrt(D), -np.inf)
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        out[:, h], size[:, h] = w @ v[:, h // G], w @ np.abs(v[:, h // G])
    e = (D + 6) * U32 * 1.4427 * (np.abs(q).max() * np.abs(k).max() * np.sqrt(D))
    return out, size * (2.0 ** -8 + 2 * e + 2 * k.shape[0] * U32) + 2.0 ** -8 * np.abs(out) + 1e-30


class Loop:
    def __init__(self, seed):
        self.g = torch.Generator().manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        n = 60
        self.k = torch.full((LAYERS, n, P, HKV, D), float("nan"), dtype=BF16, device="cuda")
        self.v = torch.full_like(self.k, float("nan"))
        self.pages = Pages(n, P)
        self.cache = PagedCache(self.k, self.v, torch.zeros((1, 20), dtype=torch.int32, device="cuda"))
        self.attention = ChunkAttention(self.cache, HQ)
        self.rows = {}                       # sequence -> (k, v) [LAYERS, t, HKV, D] on the host
        self.keep = []                       # tables of calls that may still run

    def randn(self, *shape):
        return torch.randn(shape, generator=self.g).to(BF16)

    def open(self):
        s = self.pages.open()
        self.rows[s] = (self.randn(LAYERS, 0, HKV, D), self.randn(LAYERS, 0, HKV, D))
        return s

    def grow(self, seqs, n):
        """Room for n[i] more rows, the copies that takes, and the block table."""
        copies = [c for s, m in zip(seqs, n) if (c := self.pages.resize(s, self.rows[s][0].shape[1] + m))]
        if copies:
            self.cache.copy_pages(copies)
        self.cache.table = torch.from_numpy(self.pages.block_table(seqs, 20)).cuda()
        self.keep.append(self.cache.table)

    def chunk(self, seqs, n):
        """n[i] new tokens of each sequence through both layers."""
        ctx = [self.rows[s][0].shape[1] for s in seqs]
        self.grow(seqs, n)
        chunks, total = B.make_chunks(ctx, n), sum(n)
        new = [(self.randn(LAYERS, m, HKV, D), self.randn(LAYERS, m, HKV, D)) for m in n]
        out = torch.empty((LAYERS, total, HQ, D), dtype=BF16, device="cuda")
        qs = [queries(total, HQ, D, seed=int(self.rng.integers(1 << 30))) for _ in range(LAYERS)]
        for layer in range(LAYERS):
            kk, vv = (torch.cat([x[m][layer] for x in new]).cuda() for m in range(2))
            self.cache.append(chunks, kk, vv, layer=layer)
            self.attention.run(chunks, qs[layer].cuda(), out[layer], layer=layer)
        torch.cuda.synchronize()
        q0 = 0
        for s, m, c, x in zip(seqs, n, ctx, new):
            self.rows[s] = tuple(torch.cat([a, b], 1) for a, b in zip(self.rows[s], x))
            seen = np.arange(c + m)[None] <= c + np.arange(m)[:, None]
            for layer in range(LAYERS):
                if m:
                    ref, bound = _attend(qs[layer][q0:q0 + m], self.rows[s][0][layer], self.rows[s][1][layer], seen)
                    got = out[layer, q0:q0 + m].double().cpu().numpy()
                    assert (np.abs(got - ref) <= bound).all(), (s, layer, float((np.abs(got - ref) / bound).max()))
            q0 += m

    def round(self, seqs):
        """A verified round of a random token tree per sequence."""
        parents = []
        for _ in seqs:
            m = int(self.rng.integers(1, 25))
            par = [-1] + sorted(int(self.rng.integers(0, j)) for j in range(1, m))
            parents.append([min(x, j - 1) for j, x in enumerate(par)])
        n = [len(p) for p in parents]
        ctx = [self.rows[s][0].shape[1] for s in seqs]
        self.grow(seqs, n)
        total = sum(n)
        new = [(self.randn(LAYERS, m, HKV, D), self.randn(LAYERS, m, HKV, D)) for m in n]
        kk, vv = (torch.cat([x[i] for x in new], 1).cuda() for i in range(2))
        self.cache.append(B.make_chunks(ctx, n), kk, vv)                 # every layer at once
        req = B.make_requests(ctx, tree_parents=parents)
        q = queries(total, HQ, D, seed=int(self.rng.integers(1 << 30)))
        qd, out = q.cuda(), torch.empty((total, HQ, D), dtype=F32, device="cuda")
        a, c = B.SpecAttnArgs(), self.cache.c
        a.num_q_heads, a.num_kv_heads, a.head_dim, a.dtype = HQ, HKV, D, B.SPEC_BF16
        a.q, a.out, a.q_stride_tok, a.q_stride_head = qd.data_ptr(), out.data_ptr(), HQ * D, D
        layer = 1
        a.k, a.v = self.k[layer].data_ptr(), self.v[layer].data_ptr()
        a.kv_stride_tok, a.kv_stride_head = c.kv_stride_tok, c.kv_stride_head
        a.block_table, a.block_stride, a.page_tokens, a.num_pages = c.block_table, c.block_stride, P, c.num_pages
        nd = sum(len(set(p[1:])) for p in parents)
        draft = torch.softmax(2 * torch.randn((total, VOCAB), generator=self.g), -1)
        acc = B.SpecAcceptArgs()
        acc.vocab, acc.dtype = VOCAB, B.SPEC_F32
        logits = (torch.log(draft) + 0.3 * torch.randn((total, VOCAB), generator=self.g)).cuda()
        inner, tokens = [], []
        q0 = 0
        for p in parents:                     # each child's token from its parent's row
            own = sorted(set(p[1:]))
            inner += [q0 + x for x in own]
            tokens += [int(torch.multinomial(draft[q0 + x], 1, generator=self.g)) for x in p[1:]]
            q0 += len(p)
        probs = draft[inner].contiguous().cuda() if nd else torch.zeros((1, VOCAB), device="cuda")
        tok = torch.tensor(tokens + [0], dtype=torch.int32, device="cuda")
        uni = torch.rand(total, generator=self.g).clamp_(max=1 - 2 ** -20).cuda()
        length, nxt, node = (torch.empty(len(seqs), dtype=torch.int32, device="cuda") for _ in range(3))
        acc.target_logits, acc.logits_stride = logits.data_ptr(), VOCAB
        acc.draft_probs, acc.probs_stride = probs.data_ptr(), VOCAB
        acc.draft_tokens, acc.uniforms = tok.data_ptr(), uni.data_ptr()
        acc.accepted_len, acc.next_token, acc.accepted_node = length.data_ptr(), nxt.data_ptr(), node.data_ptr()
        st, dev, host = B.spec_workspace_bytes(req, a, acc)
        B.check(st, "sizes")
        ws = torch.empty(dev + 256, dtype=torch.uint8, device="cuda")
        stage = torch.empty(host, dtype=torch.uint8, pin_memory=True)
        stream = torch.cuda.current_stream().cuda_stream
        B.check(B.spec_verify(req, a, acc, (ws.data_ptr() + 255) // 256 * 256, dev, stage.data_ptr(), host, stream),
                "spec_verify")
        self.cache.commit(req, node)          # the accepted nodes are still on the device
        torch.cuda.synchronize()
        got, q0 = out.double().cpu().numpy(), 0
        for i, s in enumerate(seqs):
            m, par = n[i], parents[i]
            seen = np.zeros((m, ctx[i] + m), bool)
            seen[:, :ctx[i]] = True
            path = {0: [0]}
            for x in range(m):
                path[x] = path[par[x]] + [x] if x else [0]
                seen[x, [ctx[i] + y for y in path[x]]] = True
            ref, bound = _attend(q[q0:q0 + m], *(torch.cat([self.rows[s][z][layer], new[i][z][layer]]) for z in range(2)),
                                 seen)
            assert (np.abs(got[q0:q0 + m] - ref) <= bound).all()
            took = path[int(node[i])]
            assert len(took) == int(length[i]) + 1
            self.rows[s] = tuple(torch.cat([self.rows[s][z], new[i][z][:, took]], 1) for z in range(2))
            assert self.pages.resize(s, self.rows[s][0].shape[1]) is None
            q0 += m
        return [int(x) for x in length]

    def check_rows(self):
        for s, (kk, vv) in self.rows.items():
            t = np.arange(kk.shape[1])
            pg = torch.from_numpy(self.pages.table(s)[t // P].astype(np.int64)).cuda()
            pl = torch.from_numpy(t % P).cuda()
            assert torch.equal(self.k[:, pg, pl].cpu(), kk) and torch.equal(self.v[:, pg, pl].cpu(), vv), s


@pytest.mark.parametrize("seed", [1, 2])
def test_prompts_forks_rounds_and_compaction(gpu_lib, seed):
    print(f"[case] serving loop {seed}", flush=True)
    w = Loop(seed)
    a, b, c = w.open(), w.open(), w.open()
    w.chunk([a, b, c], [70, 33, 1])
    w.chunk([c, a], [100, 64])                # another order, not every sequence
    w.check_rows()
    f = w.pages.fork(a)                       # shares a's pages, the last one partly filled
    w.rows[f] = w.rows[a]
    accepted = []
    for r in range(4):
        accepted += w.round([a, f, b])
        w.check_rows()
        w.chunk([c, f, b], [1, 1, 40 if r == 1 else 0])
    assert max(accepted) >= 2                 # paths that had to move
    w.pages.close(a)
    del w.rows[a]
    w.cache.copy_pages(moves) if len(moves := w.pages.compact()) else None
    w.check_rows()
    w.chunk([f, c], [5, 37])
    w.round([c, f, b])
    w.check_rows()
