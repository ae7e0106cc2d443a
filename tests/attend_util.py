"""Attention of new tokens in 64 bits with any visibility, and a bound on the
kernels' distance from it (cache_util.reference has the terms)."""
import numpy as np

from cache_util import BF16, U32


def reference(p, q, seen_of, layer=0, scale=None, out=BF16):
    """seen_of(i): bool [new tokens, rows] of request i."""
    ref, bound = [], []
    hq, d = q.shape[1], q.shape[2]
    G = hq // p.hkv
    sc = scale or 1.0 / np.sqrt(d)
    q0 = 0
    for i in range(len(p.new)):
        c, n = int(p.ctx[i]), int(p.new[i])
        kk, vv = (x[layer, :c + n].double().numpy() for x in p.rows[i])
        o, b = np.zeros((n, hq, d)), np.zeros((n, hq, d))
        seen = seen_of(i)
        for h in range(hq if n else 0):
            qq = q[q0:q0 + n, h].double().numpy()
            kh, vh = kk[:, h // G], vv[:, h // G]
            with np.errstate(invalid="ignore", over="ignore"):
                s = np.where(seen, (qq @ np.where(np.isfinite(kh), kh, 0.0).T) * sc, -np.inf)
                mag = np.where(seen, (np.abs(qq) @ np.abs(np.where(np.isfinite(kh), kh, 0.0)).T) * sc, 0.0).max(-1, keepdims=True)
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            v0 = np.where(np.isfinite(vh), vh, 0.0)
            o[:, h] = w @ v0
            size = w @ np.abs(v0)
            e = (d + 6) * U32 * 1.4427 * mag
            half = 2.0 ** -8 if out == BF16 else U32
            b[:, h] = (half + 2 * e + (2 * (c + n) + 16) * U32) * size + half * np.abs(o[:, h])
            o[:, h][(seen[:, :, None] & ~np.isfinite(vh)[None]).any(1)] = np.nan
        ref.append(o)
        bound.append(b)
        q0 += n
    return np.concatenate(ref), np.concatenate(bound) * 1.01 + 1e-30


def window_seen(p, window, sinks):
    def seen(i):
        t = int(p.ctx[i]) + np.arange(int(p.new[i]))[:, None]
        s = np.arange(int(p.ctx[i]) + int(p.new[i]))[None]
        return (s <= t) & ((s > t - window) | (s < sinks))
    return seen


def causal_seen(p):
    return window_seen(p, 1 << 40, 0)
