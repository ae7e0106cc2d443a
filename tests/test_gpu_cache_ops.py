"""GPU: rows appended to pages, accepted tree paths moved, pages copied.  These
move bytes, so every place of the pools is compared bit for bit."""
import numpy as np
import pytest
import torch

from cache_util import BF16, F32, Paged
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import Pages

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == BF16 else torch.int32).cpu()


def _same(p, want_k, want_v):
    torch.cuda.synchronize()
    assert torch.equal(_bits(p.k), _bits(want_k)) and torch.equal(_bits(p.v), _bits(want_v))


APPEND = {
    # name: ctx, new, KV heads, d, page, dtype, layers, gap between heads
    "one_row": ([0], [1], 1, 64, 32, BF16, 1, 0),
    "page_edges": ([31, 32, 33, 0, 63], [1, 1, 1, 32, 66], 2, 128, 32, BF16, 1, 0),
    "nothing_new": ([5, 100, 9], [0, 0, 3], 2, 128, 64, BF16, 1, 0),
    "layers_f32": ([10, 70], [90, 1], 3, 64, 96, F32, 5, 0),
    "odd_head_dim": ([10, 3], [9, 70], 5, 40, 64, BF16, 2, 0),
    "gaps": ([100, 3], [33, 64], 4, 128, 64, BF16, 2, 16),
    "many_requests": (list(range(300)), [1 + i % 4 for i in range(300)], 2, 64, 32, BF16, 1, 0),
    "wide_rows": ([0, 200], [5, 17], 32, 128, 64, F32, 1, 0),
}


@pytest.mark.parametrize("name", APPEND)
def test_append(gpu_lib, name):
    ctx, new, hkv, d, page, dtype, layers, gap = APPEND[name]
    print(f"[case] append {name}", flush=True)
    p = Paged(ctx, new, hkv, d, page, dtype, layers, seed=len(name), fill=3.0, gap=gap)
    p.write(p.ctx)
    k_new, v_new = p.new_rows()
    before = p.k.clone(), p.v.clone()
    p.write()
    want = p.k.clone(), p.v.clone()
    p.k.copy_(before[0])
    p.v.copy_(before[1])
    p.cache.append(p.chunks(), k_new, v_new)
    _same(p, *want)


def test_append_one_layer_from_strided_rows(gpu_lib):
    """Layer 2 of four, K and V taken from a projection's output [rows, 2, Hkv, d + 8]."""
    print("[case] append strided", flush=True)
    p = Paged([40, 0, 63], [7, 30, 64], 2, 128, 32, layers=4, seed=3, fill=1.0)
    k_new, v_new = p.new_rows()
    wide = torch.full((101, 2, 2, 136), float("nan"), dtype=BF16, device="cuda")
    wide[:, 0, :, :128], wide[:, 1, :, :128] = k_new[2], v_new[2]
    p.cache.append(p.chunks(), wide[:, 0, :, :128], wide[:, 1, :, :128], layer=2)
    want = torch.full_like(p.k, 1.0), torch.full_like(p.v, 1.0)
    q0 = 0
    for i in range(3):
        n = int(p.new[i])
        pg, pl = (torch.from_numpy(x).cuda() for x in p.where(i, np.arange(p.ctx[i], p.ctx[i] + n)))
        want[0][2, pg, pl], want[1][2, pg, pl] = k_new[2, q0:q0 + n], v_new[2, q0:q0 + n]
        q0 += n
    _same(p, *want)


def test_append_leaves_out_rows_of_bad_page_ids(gpu_lib):
    print("[case] append bad page ids", flush=True)
    p = Paged([0, 40], [70, 40], 2, 64, 32, seed=4, fill=2.0)
    k_new, v_new = p.new_rows()
    p.write()
    pg = p.table_np[0, 1]
    p.k[:, pg], p.v[:, pg] = 2.0, 2.0                    # the page whose id is lost keeps what it had
    pg1 = p.table_np[1, 2]
    p.k[:, pg1], p.v[:, pg1] = 2.0, 2.0
    place = torch.from_numpy(p.where(1, np.arange(40))[0]).cuda(), torch.from_numpy(p.where(1, np.arange(40))[1]).cuda()
    p.k[:, place[0], place[1]], p.v[:, place[0], place[1]] = 2.0, 2.0
    want = p.k.clone(), p.v.clone()
    p.k.fill_(2.0)
    p.v.fill_(2.0)
    p.table[0, 1], p.table[1, 2] = -1, p.num_pages
    p.cache.append(p.chunks(), k_new, v_new)
    _same(p, *want)


TREES = {
    "binary": [-1, 0, 0, 1, 1, 2, 2, 3, 3, 4, 4, 5, 5, 6, 6],
    "path": list(range(-1, 31)),
    "star": [-1] + [0] * 31,
    "comb": [-1, 0, 0, 2, 2, 4, 4, 6, 6, 8, 8, 10, 10, 12, 12, 14, 14, 16, 16, 18, 18],
    "one": [-1],
}


def _path(par, node):
    at = [node]
    while par[at[-1]] >= 0:
        at.append(par[at[-1]])
    return at[::-1]


def _commit_case(ctx, parents, nodes, hkv, d, page, dtype, layers, shared, gap=0):
    p = Paged(ctx, [len(x) for x in parents], hkv, d, page, dtype, layers, seed=len(ctx), fill=5.0, gap=gap).write()
    want = p.k.clone(), p.v.clone()
    for i, (par, node) in enumerate(zip(parents, nodes)):
        if not 0 <= node < len(par):
            continue
        path = _path(par, node)
        dst, src = p.where(i, ctx[i] + np.arange(len(path))), p.where(i, ctx[i] + np.array(path))
        for w, pool in zip(want, (p.k, p.v)):
            w[:, torch.from_numpy(dst[0]).cuda(), torch.from_numpy(dst[1]).cuda()] = \
                pool[:, torch.from_numpy(src[0]).cuda(), torch.from_numpy(src[1]).cuda()]
    req = B.make_requests(ctx, None, parents[0]) if shared else B.make_requests(ctx, tree_parents=parents)
    p.cache.commit(req, torch.tensor(nodes, dtype=torch.int32, device="cuda"))
    _same(p, *want)


@pytest.mark.parametrize("name", TREES)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_commit_every_node_of_a_shared_tree(gpu_lib, name, dtype):
    print(f"[case] commit {name} {dtype}", flush=True)
    par = TREES[name]
    n = len(par)
    nodes = list(range(n)) + [-1, n]                     # and two that are no nodes
    ctx = [(7 * i) % 70 for i in range(len(nodes))]
    _commit_case(ctx, [par] * len(nodes), nodes, 2, 64, 32, dtype, 3, True)


def test_commit_trees_of_their_own(gpu_lib):
    """More requests than one launch holds, random trees, gaps between heads."""
    print("[case] commit own trees", flush=True)
    rng = np.random.default_rng(2)
    parents, nodes, ctx = [], [], []
    for _ in range(150):
        n = int(rng.integers(1, 33))
        par = [-1] + sorted(int(rng.integers(0, j)) for j in range(1, n))
        par = [min(x, j - 1) for j, x in enumerate(par)]
        parents.append(par)
        nodes.append(int(rng.integers(-1, n)))
        ctx.append(int(rng.integers(0, 100)))
    _commit_case(ctx, parents, nodes, 3, 128, 64, BF16, 2, False, gap=8)


def test_commit_of_chains_changes_nothing(gpu_lib):
    print("[case] commit chains", flush=True)
    p = Paged([10, 60], [5, 3], 2, 64, 32, seed=1, fill=0.0).write()
    want = p.k.clone(), p.v.clone()
    p.cache.commit(B.make_requests([10, 60], [4, 2]), torch.tensor([2, 0], dtype=torch.int32, device="cuda"))
    _same(p, *want)


@pytest.mark.parametrize("n,page,hkv,d,dtype,layers,gap", [
    (1, 32, 1, 64, BF16, 1, 0), (7, 96, 3, 64, F32, 3, 0), (300, 32, 2, 64, BF16, 2, 0), (5, 64, 4, 128, BF16, 2, 24),
    (2, 256, 8, 128, BF16, 1, 0)])
def test_copy_pages(gpu_lib, n, page, hkv, d, dtype, layers, gap):
    print(f"[case] copy pages {n} {page}", flush=True)
    rng = np.random.default_rng(n)
    pages = 2 * n + 5
    p = Paged([pages * page], [0], hkv, d, page, dtype, layers, seed=n, spare=0, gap=gap).write()
    order = rng.permutation(pages).astype(np.int32)
    # a page may be the source of several copies
    pairs = np.stack([order[:n], order[n:2 * n], rng.integers(1, page + 1, n)], 1)
    pairs[:, 0] = np.where(rng.random(n) < 0.3, pairs[0, 0], pairs[:, 0])
    want = p.k.clone(), p.v.clone()
    for s, t, rows in pairs.tolist():
        want[0][:, t, :rows], want[1][:, t, :rows] = p.k[:, s, :rows], p.v[:, s, :rows]
    p.cache.copy_pages(pairs)
    _same(p, *want)


def test_movers_past_4_gib_and_in_a_graph(gpu_lib):
    """Appended, committed and copied rows at the end of pools of over 4 GiB,
    eagerly and replayed (what the host gave stays in the captured launches)."""
    row = 2 * 128 * 2
    spare = (1 << 32) // (64 * row) + 100
    print("[case] movers past 4 GiB", flush=True)
    par = TREES["binary"]
    p = Paged([70, 5], [15, 15], 2, 128, spare=spare, far=True, seed=3, fill=0.0)
    p.write(p.ctx)
    k_new, v_new = p.new_rows()
    chunks, req = p.chunks(), B.make_requests([70, 5], None, par)
    node = torch.tensor([13, 9], dtype=torch.int32, device="cuda")
    used = sorted(set(p.table_np[0, :2].tolist() + p.table_np[1, :1].tolist()))
    copies = [[used[0], 3, 64], [used[1], 1, 11]]

    def call():
        p.cache.append(chunks, k_new, v_new)
        p.cache.commit(req, node)
        p.cache.copy_pages(copies)

    look = used + [1, 3]
    call()
    torch.cuda.synchronize()
    want = p.k[:, look].clone(), p.v[:, look].clone()
    q0 = 0
    for i, nd in enumerate([13, 9]):
        for t, x in enumerate(_path(par, nd)):
            pg, pl = p.where(i, int(p.ctx[i]) + t)
            assert torch.equal(p.k[0, int(pg), int(pl)], k_new[0, q0 + x])
        q0 += 15
    assert torch.equal(p.v[0, 3], p.v[0, used[0]]) and torch.equal(p.v[0, 1, :11], p.v[0, used[1], :11])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    chunks.ctx_len[0] = 0                                # a replay does not look at the host's arrays again
    for _ in range(3):
        p.k[:, look], p.v[:, look] = 0.0, 0.0
        p.k[:, 1], p.k[:, 3] = 0.0, 0.0
        keep = p.k[:, used[0]].clone()
        g.replay()
        torch.cuda.synchronize()
        for i, nd in enumerate([13, 9]):
            for t, x in enumerate(_path(par, nd)):
                pg, pl = p.where(i, [70, 5][i] + t)
                assert torch.equal(p.k[0, int(pg), int(pl)], k_new[0, 15 * i + x])
        del keep
    del p, want, g
    torch.cuda.empty_cache()


def test_fork_and_compaction_keep_every_sequence(gpu_lib):
    """Sequences grow, fork, shrink and close; the copies that the bookkeeping
    asks for are made; every sequence still reads its own rows."""
    print("[case] pages and copies", flush=True)
    P, hkv, d, layers = 32, 2, 64, 2
    rng = np.random.default_rng(11)
    pages = Pages(60, P)
    k = torch.zeros((layers, 60, P, hkv, d), dtype=F32, device="cuda")
    v = torch.zeros_like(k)
    from paper_2505_17074_amd.cache import PagedCache
    cache = PagedCache(k, v, torch.zeros((1, 60), dtype=torch.int32, device="cuda"))
    rows = {}                                            # the model: each sequence's row values

    def grow(s, n):
        old = len(rows[s])
        c = pages.resize(s, old + n)
        if c:
            cache.copy_pages([c])
        vals = rng.standard_normal(n).astype(np.float32)
        cache.table = torch.from_numpy(pages.block_table([s])).cuda()
        x = torch.from_numpy(vals).cuda()[None, :, None, None].expand(layers, n, hkv, d).contiguous()
        cache.append(B.make_chunks([old], [n]), x, -x)
        rows[s] = np.concatenate([rows[s], vals])

    for step in range(120):
        what = rng.choice(["open", "grow", "grow", "grow", "fork", "fork", "shrink", "close", "compact"])
        live = sorted(rows)
        if what == "open" or not live:
            s = pages.open()
            rows[s] = np.zeros(0, np.float32)
        elif what == "grow":
            s, n = int(rng.choice(live)), int(rng.integers(1, 70))
            if pages.free >= n // P + 3:
                grow(s, n)
        elif what == "fork":
            s = int(rng.choice(live))
            rows[pages.fork(s)] = rows[s].copy()
        elif what == "shrink":
            s = int(rng.choice(live))
            n = int(rng.integers(0, len(rows[s]) + 1))
            assert pages.resize(s, n) is None
            rows[s] = rows[s][:n]
        elif what == "close" and len(live) > 2:
            s = int(rng.choice(live))
            pages.close(s)
            del rows[s]
        elif what == "compact":
            c = pages.compact()
            if len(c):
                cache.copy_pages(c)
            used = 60 - pages.free
            assert all((pages.table(s) < used).all() for s in rows)
        if step % 10 == 9:
            torch.cuda.synchronize()
            for s, r in rows.items():
                t = torch.from_numpy(pages.table(s)).long().cuda()
                got = k[1, t].reshape(-1, hkv, d)[:len(r), 1, 5].cpu().numpy()
                assert np.array_equal(got, r), (step, s)
                assert np.array_equal(-v[0, t].reshape(-1, hkv, d)[:len(r), 0, 63].cpu().numpy(), r)


@pytest.mark.parametrize("ctx,new,hkv,d,page,dtype,layers,gap", [
    (0, 700, 2, 128, 64, BF16, 2, 0), (37, 1, 2, 64, 32, F32, 3, 0), (47, 18, 3, 40, 96, BF16, 1, 8),
    (1000, 5, 8, 128, 64, BF16, 2, 0), (15, 1, 1, 64, 32, BF16, 1, 0)])
def test_append_of_one_request(gpu_lib, ctx, new, hkv, d, page, dtype, layers, gap):
    """Alone, and among others that have nothing new."""
    print(f"[case] append one request {ctx} {new}", flush=True)
    p = Paged([3, ctx, 9], [0, new, 0], hkv, d, page, dtype, layers, seed=ctx + new, fill=3.0, gap=gap)
    p.write(p.ctx)
    k_new, v_new = p.new_rows()
    before = p.k.clone(), p.v.clone()
    p.write()
    want = p.k.clone(), p.v.clone()
    table = p.table
    for chunks, rows in ((p.chunks(), table), (B.make_chunks([ctx], [new]), table[1:2])):
        p.k.copy_(before[0])
        p.v.copy_(before[1])
        p.cache.table = rows
        p.cache.append(chunks, k_new, v_new)
        _same(p, *want)


@pytest.mark.parametrize("shared", [True, False], ids=["shared", "own"])
@pytest.mark.parametrize("n,node", [(1, 0), (2, 1), (32, 31), (32, 17), (15, -1)])
def test_commit_of_one_tree(gpu_lib, n, node, shared):
    print(f"[case] commit one tree {n} {node}", flush=True)
    rng = np.random.default_rng(n + node)
    par = [-1] + [int(rng.integers(max(0, j - 3), j)) for j in range(1, n)]
    _commit_case([29], [par], [node], 2, 128, 32, BF16, 2, shared)


@pytest.mark.parametrize("n", [4, 5, 6])
def test_copies_of_a_few_pages(gpu_lib, n):
    print(f"[case] copy {n} pages", flush=True)
    p = Paged([64 * 20], [0], 2, 128, 64, layers=2, seed=n, spare=0).write()
    pairs = np.array([[i, 19 - i, 64 - 9 * i] for i in range(n)], np.int32)
    want = p.k.clone(), p.v.clone()
    for s, t, rows in pairs.tolist():
        want[0][:, t, :rows], want[1][:, t, :rows] = p.k[:, s, :rows], p.v[:, s, :rows]
    p.cache.copy_pages(pairs)
    _same(p, *want)
