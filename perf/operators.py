"""The paged cache's operators: what a serving loop does with the cache around
the verify step, in plain torch (own = False) and through the library's entry
points (own = True).

Four kinds of pass ("op"):
  chunk   attention of each request's new tokens over its paged cache, one layer
  append  new K/V rows into the pages, one layer or all of them
  round   a verified round's bookkeeping over all layers: the token trees' rows
          appended, then the accepted paths' rows moved behind their contexts
  pages   pages (or their first rows) copied to other pages, all layers

A case holds sizes only.  Lengths come from its "mix", values from the seed.
"""
import math

import numpy as np
import torch

own = False

_DEV = "cuda"
_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, batch, **kw):
    c = {"op": op, "batch": batch, "mix": 0, "layers": 1, "hkv": 8, "d": 128, "page": 64, "dtype": "bf16"}
    if name:
        c["name"] = name
    if op == "chunk":
        c.update(hq=32, ctx_lo=0, ctx_hi=0, new_lo=1, new_hi=1, ones=0, out="bf16")
    elif op == "append":
        c.update(ctx_lo=0, ctx_hi=0, new_lo=1, new_hi=1)
    elif op == "round":
        c.update(ctx_lo=0, ctx_hi=0, nodes=15, tree="binary")
    c.update(kw)
    return c


def listed():
    return [
        # one interactive request decoding a token over a kilotoken: latency
        _case("chunk_one_token_b1", "chunk", 1, ctx_lo=1000, ctx_hi=1000),
        # decoding: a token each over ragged contexts, bound by the cache's bytes
        _case("chunk_decode_b64", "chunk", 64, ctx_lo=512, ctx_hi=8192),
        # a prompt's first chunk, nothing cached yet
        _case("chunk_prompt_b1", "chunk", 1, new_lo=2048, new_hi=2048),
        # continuous batching: prompts' chunks of odd lengths among decoding requests, MHA heads
        _case("chunk_mixed_b24", "chunk", 24, hkv=32, ctx_lo=100, ctx_hi=2500, new_lo=33, new_hi=700, ones=16, page=32),
        # a small model's heads, fp32 output as the verify attention writes it
        _case("chunk_ragged_d64_b16", "chunk", 16, hq=16, hkv=4, d=64, ctx_hi=1500, new_lo=1, new_hi=400, page=96, out="f32"),
        # a long prompt's last chunk: wide GQA groups, 30 thousand rows cached
        _case("chunk_long_b1", "chunk", 1, hq=64, ctx_lo=30011, ctx_hi=30011, new_lo=1024, new_hi=1024),
        # a verify round's new rows of one layer, many ragged requests
        _case("append_verify_b128", "append", 128, ctx_lo=32, ctx_hi=900, new_lo=2, new_hi=9),
        # a prompt's rows of every layer at once (a cache brought in from elsewhere)
        _case("append_layers_b4", "append", 4, layers=32, ctx_hi=200, new_lo=300, new_hi=700),
        # the cache after a round of one request's tree
        _case("round_tree_b1", "round", 1, layers=32, ctx_lo=777, ctx_hi=777),
        # the cache after a round of binary token trees, 32 layers
        _case("round_tree15_b64", "round", 64, layers=32, ctx_lo=100, ctx_hi=170),
        # copy on write of one forked request's last, partly filled page
        _case("pages_fork_b1", "pages", 1, layers=32),
        # compaction: many whole pages move
        _case("pages_compact_b96", "pages", 96, layers=32, whole=1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["chunk", "chunk", "chunk", "append", "round", "pages"])
    kw = {"mix": rng.randint(1, 1 << 20), "page": rng.choice([32, 64, 96, 128, 256])}
    if op == "chunk":
        hq, hkv, d = rng.choice([(32, 8, 128), (32, 32, 128), (64, 8, 128), (8, 8, 64), (16, 4, 64), (12, 4, 128), (8, 1, 128)])
        new_hi = rng.choice([1, _log_int(rng, 2, 40), _log_int(rng, 40, 2048), _log_int(rng, 40, 2048)])
        ctx_hi = _log_int(rng, 16, 30000)
        batch = _log_int(rng, 1, 64)
        while batch * hq * new_hi * (ctx_hi + new_hi) > 1.5e9 or batch * (ctx_hi + new_hi) * hkv * d > 4e8:
            if batch > 1:
                batch = batch // 2
            elif new_hi > 256:
                new_hi = new_hi // 2
            else:
                ctx_hi = ctx_hi // 2
        kw.update(hq=hq, hkv=hkv, d=d, ctx_lo=rng.choice([0, ctx_hi // 2, ctx_hi]), ctx_hi=ctx_hi, new_hi=new_hi,
                  new_lo=max(1, new_hi // rng.choice([1, 3, 1000])), ones=rng.choice([0, batch // 2]),
                  out=rng.choice(["bf16", "bf16", "f32"]))
        return _case("", op, batch, **kw)
    hkv, d = rng.choice([(8, 128), (32, 128), (4, 64), (8, 64)])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    layers = rng.choice([1, 4, 32])
    room = 300_000_000 // (layers * hkv * d * (4 if dtype == "f32" else 2))    # rows of K in 300 MB
    kw.update(hkv=hkv, d=d, dtype=dtype, layers=layers)
    if op == "pages":
        n = _log_int(rng, 1, 96)
        return _case("", op, max(1, min(n, room // (2 * kw["page"]) - 2)), whole=rng.choice([0, 1]), **kw)
    ctx = _log_int(rng, 1, 1000)
    new = rng.randint(2, 32) if op == "round" else _log_int(rng, 1, 700)
    batch = max(1, min(_log_int(rng, 1, 128), room // (ctx + new + kw["page"])))
    kw.update(ctx_lo=ctx // rng.choice([1, 4]), ctx_hi=ctx)
    if op == "round":
        kw.update(nodes=new, tree=rng.choice(["binary", "random"]))
    else:
        kw.update(new_lo=max(1, new // rng.choice([1, 4])), new_hi=new)
    return _case("", op, batch, **kw)


# ---- shapes of a case ------------------------------------------------------
def _lengths(c):
    """Cached and new rows of each request (the first `ones` decode a token)."""
    rng = np.random.default_rng([c["mix"], c["batch"]])
    ctx = rng.integers(c["ctx_lo"], c["ctx_hi"] + 1, c["batch"])
    if c["op"] == "round":
        return ctx, np.full(c["batch"], c["nodes"], np.int64)
    new = rng.integers(c["new_lo"], c["new_hi"] + 1, c["batch"])
    new[:c.get("ones", 0)] = 1
    order = rng.permutation(c["batch"])
    return ctx[order], new[order]


def _tree(c):
    """BFS parents of the trees' common topology."""
    n = c["nodes"]
    if c["tree"] == "binary":
        return (np.arange(n) - 1) // 2
    rng = np.random.default_rng([c["mix"], n, 5])
    return np.array([-1] + sorted(int(rng.integers(0, j)) for j in range(1, n)), np.int64).clip(max=np.arange(-1, n - 1))


def _path(par, node):
    at = [int(node)]
    while par[at[-1]] >= 0:
        at.append(int(par[at[-1]]))
    return at[::-1]


def _accepted(c):
    rng = np.random.default_rng([c["mix"], c["nodes"], 9])
    return rng.integers(0, c["nodes"], c["batch"]).astype(np.int32)


def _copied(c):
    """Rows of each copied page: whole pages, or a fork's partly filled last one."""
    rng = np.random.default_rng([c["mix"], c["batch"], 3])
    return np.full(c["batch"], c["page"]) if c.get("whole") else rng.integers(1, c["page"] + 1, c["batch"])


def work(case):
    c = case
    row = c["hkv"] * c["d"] * (4 if c["dtype"] == "f32" else 2) * 2 * c["layers"]     # a token's K and V, all layers
    if c["op"] == "pages":
        return {"bytes": 2 * row * int(_copied(c).sum()), "flops": 0}
    ctx, new = _lengths(c)
    if c["op"] == "append":
        return {"bytes": 2 * row * int(new.sum()), "flops": 0}
    if c["op"] == "round":
        # the rows appended, then the nodes of the path that are not in their place yet
        par = _tree(c)
        moved = sum(sum(x != t for t, x in enumerate(_path(par, a))) for a in _accepted(c))
        return {"bytes": 2 * row * (int(new.sum()) + moved), "flops": 0}
    out = int(new.sum()) * c["hq"] * c["d"] * (2 + (4 if c["out"] == "f32" else 2))
    seen = int((new * ctx + new * (new + 1) // 2).sum())
    return {"bytes": row * int((ctx + new).sum()) + out, "flops": 4 * c["d"] * c["hq"] * seen}


# ---- inputs ----------------------------------------------------------------
class _State:
    pass


def _inputs(c, seed):
    """The pools hold random rows throughout: a page is never clean of what the
    requests before left in it."""
    s = _State()
    s.case = c
    g = torch.Generator(device=_DEV)
    g.manual_seed(int(seed) * 6151 + 29)
    dt, P, L, hkv, d, b = _DTYPE[c["dtype"]], c["page"], c["layers"], c["hkv"], c["d"], c["batch"]
    randn = lambda *shape: torch.randn(shape, generator=g, device=_DEV, dtype=dt)  # noqa: E731
    if c["op"] == "pages":
        total = 2 * b
    else:
        s.ctx, s.new = _lengths(c)
        s.first = np.concatenate([[0], np.cumsum(s.new)])
        pages = -(-(s.ctx + s.new) // P)
        total = int(pages.sum())
    s.num_pages = total + 3
    order = torch.randperm(s.num_pages, generator=g, device=_DEV)[:total].to(torch.int32)
    s.k, s.v = randn(L, s.num_pages, P, hkv, d), randn(L, s.num_pages, P, hkv, d)
    if c["op"] == "pages":
        s.rows = _copied(c)
        s.pairs = np.stack([order[:b].cpu().numpy(), order[b:].cpu().numpy(), s.rows], 1).astype(np.int32)
        s.table = None
        return s
    at = np.concatenate([[0], np.cumsum(pages)])
    pick = np.minimum(at[:-1, None] + np.arange(int(pages.max())), at[1:, None] - 1)
    s.table = order[torch.from_numpy(pick).to(_DEV)].contiguous()
    s.ctx_dev, s.new_dev = torch.from_numpy(s.ctx).to(_DEV), torch.from_numpy(s.new).to(_DEV)
    s.first_dev = torch.from_numpy(s.first).to(_DEV)
    n = int(s.new.sum())
    s.owner = torch.from_numpy(np.repeat(np.arange(b), s.new)).to(_DEV)        # request of each new token
    s.place = torch.arange(n, device=_DEV) - s.first_dev[s.owner]              # and its place among the request's
    if c["op"] == "chunk":
        s.q = randn(n, c["hq"], d)
        s.out = torch.empty((n, c["hq"], d), dtype=_DTYPE[c["out"]], device=_DEV)
    else:
        s.k_new, s.v_new = randn(L, n, hkv, d), randn(L, n, hkv, d)
    if c["op"] == "round":
        par = _tree(c)
        s.parents = par.astype(np.int32)
        s.accepted = torch.from_numpy(_accepted(c)).to(_DEV)
        depth = max(len(_path(par, x)) for x in range(c["nodes"]))
        paths = np.array([(_path(par, x) + [-1] * depth)[:depth] for x in range(c["nodes"])])
        s.paths = torch.from_numpy(paths).to(_DEV)                             # the topology's paths, -1 behind their ends
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2505_17074_amd import binding as B
        from paper_2505_17074_amd.cache import ChunkAttention, PagedCache
        s.cache = PagedCache(s.k, s.v, s.table)
        if case["op"] != "pages":
            s.chunks = B.make_chunks(s.ctx, s.new)
        if case["op"] == "chunk":
            s.attention = ChunkAttention(s.cache, case["hq"])
        elif case["op"] == "round":
            s.requests = B.make_requests(s.ctx, None, s.parents)
    return s


# ---- the plain forms -------------------------------------------------------
def _pool_rows(s, request, position):
    """Pool row (page x page size + place) of the requests' positions."""
    P = s.case["page"]
    return s.table[request, position // P].long() * P + position % P


def _chunk(s):
    """Every request padded to the longest: gather, scores, softmax, product in 32 bits."""
    c = s.case
    b, hq, hkv, d = c["batch"], c["hq"], c["hkv"], c["d"]
    G, n, length = hq // hkv, int(s.new.max()), int((s.ctx + s.new).max())
    t = torch.arange(length, device=_DEV)
    j = torch.arange(n, device=_DEV)
    total = s.ctx_dev + s.new_dev
    rows = _pool_rows(s, torch.arange(b, device=_DEV)[:, None], torch.minimum(t[None], total[:, None] - 1))
    k = s.k.view(-1, hkv, d)[rows].float().permute(0, 2, 3, 1).contiguous()            # [b, hkv, d, length]
    v = s.v.view(-1, hkv, d)[rows].float().permute(0, 2, 1, 3).contiguous()            # [b, hkv, length, d]
    mine = s.first_dev[:-1, None] + torch.minimum(j[None], s.new_dev[:, None] - 1)
    q = s.q[mine].float().view(b, n, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, G * n, d).contiguous()
    x = torch.matmul(q, k).view(b, hkv, G, n, length)
    x = x.mul_(1.0 / math.sqrt(d))
    seen = t[None, None] <= s.ctx_dev[:, None, None] + j[None, :, None]
    x = x.masked_fill_(~seen[:, None, None], float("-inf"))
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    x = x.div_(x.sum(-1, keepdim=True))
    o = torch.matmul(x.view(b, hkv, G * n, length), v).view(b, hkv, G, n, d)
    o = o.permute(0, 3, 1, 2, 4).reshape(b, n, hq, d)
    s.out.copy_(o[s.owner, s.place])
    return s.out


def _append(s):
    rows = _pool_rows(s, s.owner, s.ctx_dev[s.owner] + s.place)
    L, hkv, d = s.k.shape[0], s.case["hkv"], s.case["d"]
    s.k.view(L, -1, hkv, d)[:, rows] = s.k_new
    s.v.view(L, -1, hkv, d)[:, rows] = s.v_new
    return {"k": s.k, "v": s.v}


def _move(s, src, dst):
    L, hkv, d = s.k.shape[0], s.case["hkv"], s.case["d"]
    for pool in (s.k.view(L, -1, hkv, d), s.v.view(L, -1, hkv, d)):
        pool[:, dst] = pool[:, src]           # the right side is gathered whole before the left is written


def _round(s):
    _append(s)
    path = s.paths[s.accepted.long()]                                                  # [b, depth]
    request, t = torch.nonzero(path >= 0, as_tuple=True)
    ctx = s.ctx_dev[request]
    _move(s, _pool_rows(s, request, ctx + path[request, t]), _pool_rows(s, request, ctx + t))
    return {"k": s.k, "v": s.v}


def _pages(s):
    P = s.case["page"]
    pairs = torch.from_numpy(s.pairs).to(_DEV).long()
    pair, t = torch.nonzero(torch.arange(P, device=_DEV)[None] < pairs[:, 2:], as_tuple=True)
    _move(s, pairs[pair, 0] * P + t, pairs[pair, 1] * P + t)
    return {"k": s.k, "v": s.v}


def run(state):
    s = state
    op = s.case["op"]
    if not own:
        return {"chunk": _chunk, "append": _append, "round": _round, "pages": _pages}[op](s)
    if op == "chunk":
        s.attention.run(s.chunks, s.q, s.out)
        return s.out
    if op == "pages":
        s.cache.copy_pages(s.pairs)
    else:
        s.cache.append(s.chunks, s.k_new, s.v_new)
        if op == "round":
            s.cache.commit(s.requests, s.accepted)
    return {"k": s.k, "v": s.v}


# ---- the same outputs from the definitions, in 64 bits ----------------------
def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["op"] != "chunk":
        return {"k": _copies(s, s.k, s.__dict__.get("k_new")), "v": _copies(s, s.v, s.__dict__.get("v_new"))}
    G, d = c["hq"] // c["hkv"], c["d"]
    out = torch.zeros(s.out.shape, dtype=torch.float64, device=_DEV)
    for i in range(c["batch"]):
        ctx, n, q0 = int(s.ctx[i]), int(s.new[i]), int(s.first[i])
        pages = s.table[i].long()[:-(-(ctx + n) // c["page"])]
        for h in range(c["hkv"]):
            k = s.k[0, pages, :, h].reshape(-1, d)[:ctx + n].double()
            v = s.v[0, pages, :, h].reshape(-1, d)[:ctx + n].double()
            for g in range(h * G, (h + 1) * G):
                x = torch.mm(s.q[q0:q0 + n, g].double(), k.t().contiguous()) / d ** 0.5
                x[torch.ones_like(x, dtype=torch.bool).triu_(ctx + 1)] = float("-inf")
                out[q0:q0 + n, g] = torch.mm(torch.softmax(x, -1), v)
    return out


def _copies(s, pool, fresh):
    """A pool after the pass, a page or a request's rows at a time (copies are
    exact in any type)."""
    c, P = s.case, s.case["page"]
    before = pool.clone()
    if c["op"] == "pages":
        for src, dst, n in s.pairs.tolist():
            pool[:, dst, :n] = before[:, src, :n]
        return pool
    table = s.table.cpu().numpy()
    for i in range(c["batch"]):
        ctx, n, first = int(s.ctx[i]), int(s.new[i]), int(s.first[i])
        t = np.arange(ctx, ctx + n)
        page, place = (torch.from_numpy(x).long().to(_DEV) for x in (table[i, t // P], t % P))
        rows = fresh[:, first:first + n]
        if c["op"] == "round":          # the path's rows in front, the others where they were
            path = _path(_tree(c), int(s.accepted[i]))
            rows = rows[:, path + list(range(len(path), n))]
        pool[:, page, place] = rows
    return pool
