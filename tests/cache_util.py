"""Paged caches for the tests: pools whose every unused place is NaN, a
shuffled block table, and the operators' definitions in 64 bits (numpy)."""
import numpy as np
import torch

from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import PagedCache

BF16, F32 = torch.bfloat16, torch.float32


class Paged:
    """ctx + new rows of each request in shuffled pages [layers, pages, P, Hkv, d];
    `fill` elsewhere.  k, v: the rows as fp64 [layers][request] arrays."""

    def __init__(self, ctx, new, hkv, d, page=64, dtype=BF16, layers=1, seed=0, spare=3, fill=float("nan"),
                 device="cuda", gap=0, far=False):
        self.ctx, self.new = np.asarray(ctx, np.int64), np.asarray(new, np.int64)
        self.page, self.hkv, self.d, self.layers, self.dtype = page, hkv, d, layers, dtype
        rng = np.random.default_rng(seed)
        total = self.ctx + self.new
        pages = -(-total // page)
        used = int(pages.sum())
        self.num_pages = used + spare
        # far: the pages at the pool's end
        ids = np.arange(self.num_pages - used, self.num_pages) if far else np.arange(self.num_pages)
        order = rng.permutation(ids)[:used].astype(np.int32)
        self.table_np = np.full((len(total), int(pages.max())), -7, np.int32)   # never read behind a request's pages
        at = 0
        for i, n in enumerate(pages):
            self.table_np[i, :n] = order[at:at + n]
            at += n
        shape = (layers, self.num_pages, page, hkv, d + gap)
        self.k, self.v = (torch.full(shape, fill, dtype=dtype, device=device)[..., :d] for _ in range(2))
        self.rows = []
        g = torch.Generator().manual_seed(int(seed) + 1)
        for i in range(len(total)):
            kk, vv = (torch.randn((layers, int(total[i]), hkv, d), generator=g).to(dtype) for _ in range(2))
            self.rows.append((kk, vv))
        self.table = torch.from_numpy(self.table_np).to(device)
        self.cache = PagedCache(self.k, self.v, self.table)
        self.device = device

    def where(self, i, t):
        """(page, place) of request i's rows t."""
        t = np.asarray(t, np.int64)
        return self.table_np[i, t // self.page].astype(np.int64), t % self.page

    def write(self, upto=None):
        """The requests' rows (the first upto[i] of them) into the pools."""
        for i, (kk, vv) in enumerate(self.rows):
            n = kk.shape[1] if upto is None else int(upto[i])
            if n:
                pg, pl = (torch.from_numpy(x).to(self.device) for x in self.where(i, np.arange(n)))
                self.k[:, pg, pl] = kk[:, :n].to(self.device)
                self.v[:, pg, pl] = vv[:, :n].to(self.device)
        return self

    def chunks(self):
        return B.make_chunks(self.ctx, self.new)

    def new_rows(self, extra=0):
        """The new rows packed [layers, Nq, Hkv, d]."""
        out = []
        for m in range(2):
            x = [r[m][:, int(c):] for r, c in zip(self.rows, self.ctx)]
            out.append(torch.cat(x, 1).to(self.device))
        return out


def queries(n, hq, d, seed=0, dtype=BF16):
    return torch.randn((n, hq, d), generator=torch.Generator().manual_seed(int(seed) + 5)).to(dtype)


U32 = 2.0 ** -24


def reference(p: Paged, q, layer=0, scale=None, out=BF16):
    """The definition in 64 bits and a bound on the kernels' distance from it,
    per element:
      scores: d products summed in fp32, then scale and the subtraction of the
        reference, each at most half a step of their terms' size: an absolute
        error e of the exponent, a relative error of about e of a weight;
      weights: exp2 (a step), a bf16 weight half a step, 2^-8 (in three parts
        2^-24); sums of L terms, L 2^-24 at most, for the products and for the
        normaliser, and another for joined pieces;
      the output's own rounding: half a step."""
    ref, bound = [], []
    hq, d = q.shape[1], q.shape[2]
    G = hq // p.hkv
    sc = scale or 1.0 / np.sqrt(d)
    q0 = 0
    for i in range(len(p.new)):
        c, n = int(p.ctx[i]), int(p.new[i])
        kk, vv = (x[layer, :c + n].double().numpy() for x in p.rows[i])
        o, b = np.zeros((n, hq, d)), np.zeros((n, hq, d))
        for h in range(hq):
            qq = q[q0:q0 + n, h].double().numpy()
            kh, vh = kk[:, h // G], vv[:, h // G]
            seen = np.arange(c + n)[None] <= c + np.arange(n)[:, None]
            with np.errstate(invalid="ignore", over="ignore"):
                s = np.where(seen, (qq @ kh.T) * sc, -np.inf)
                mag = np.where(seen, (np.abs(qq) @ np.abs(kh).T) * sc, 0.0).max(-1, keepdims=True)
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            v0 = np.where(np.isfinite(vh), vh, 0.0)
            o[:, h] = w @ v0
            bad = (seen[:, :, None] & ~np.isfinite(vh)[None]).any(1) if not np.isfinite(vh).all() else None
            size = w @ np.abs(v0)
            e = (d + 6) * U32 * 1.4427 * mag
            part = (2.0 ** -8 if out == BF16 else U32) + 2 * e + (2 * (c + n) + 16) * U32
            b[:, h] = part * size + (2.0 ** -8 if out == BF16 else U32) * np.abs(o[:, h])
            if bad is not None:
                o[:, h][bad] = np.nan
        ref.append(o)
        bound.append(b)
        q0 += n
    return np.concatenate(ref), np.concatenate(bound) * 1.01 + 1e-30


def check_close(got, ref, bound):
    got = got.double().cpu().numpy()
    fine = np.isfinite(ref)
    assert not np.isfinite(got[~fine]).any()
    off = np.abs(got - ref)[fine] / bound[fine]
    assert np.isfinite(got[fine]).all()
    assert off.size == 0 or off.max() <= 1.0, float(off.max())
