"""GPU: sampled rows whose border is near a sum as well as all others: the token
is one that a row may have, its distribution is one, its kept logits are the
logits.  Long batches, and rows whose unmasked tokens lie beside each other."""
import numpy as np
import pytest
import torch

from paper_2505_17074_amd.sample import Sampler
from test_gpu_sample import BF16, F32, FILTERS, PROB, _check, _f, _filters, _i, _logits, _run

pytestmark = pytest.mark.gpu


def _holds(logits, tokens, T=None, probs=None, kept=None, one=None):
    """What is so of every row, however near its sums are to their borders.  one:
    the rows of the first token alone."""
    V = logits.shape[1]
    x = logits.double().cpu().numpy()
    half = 2.0 ** -8 if logits.dtype == BF16 else 2.0 ** -24
    for i in range(x.shape[0]):
        t = tokens[i].item()
        assert 0 <= t < V and x[i, t] > -np.inf, (i, t)
        if probs is not None:
            got = probs[i].double().cpu().numpy()
            assert np.isfinite(got).all() and (got >= 0).all() and got[t] > 0, i
            assert (got[~(x[i] > -np.inf)] == 0).all(), i
            # each is rounded by half a step of its own, or of the smallest normal number
            assert abs(got.sum() - 1) <= half * 1.001 + PROB + V * 2.0 ** -126, i
        if kept is not None:
            got = kept[i].double().cpu().numpy()
            stays = got != torch.finfo(logits.dtype).min
            assert stays[t] and (x[i][stays] > -np.inf).all(), i
            temp = 1.0 if T is None else T[i].item()
            want = np.zeros(stays.sum()) if one is not None and one[i] else x[i][stays] / temp
            assert (np.abs(got[stays] - want) <= np.abs(want) * half * 1.001 + 2.0 ** -126).all(), i
            # what stays is a run of the order: nothing above it was left out
            assert not (x[i][~stays] > x[i][stays].min()).any(), i


@pytest.mark.parametrize("kind", ["probs", "kept_logits"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 1000, 4099, 32000, 50257, 128256])
@pytest.mark.parametrize("name", FILTERS)
def test_every_row(gpu_lib, name, V, dtype, kind):
    print(f"[case] sample every row {name} {V} {dtype} {kind}", flush=True)
    kw = _filters(name)
    x, u = _logits(5, V, dtype, seed=V + len(name) + 1000)
    tokens, out = _run(x, u, kind, **kw)
    T = kw.get("temperature")
    _holds(x, tokens, T, probs=out if kind == "probs" else None, kept=out if kind == "kept_logits" else None,
           one=None if T is None else [not t > 0 for t in T.tolist()])


@pytest.mark.parametrize("kind", [None, "probs", "kept_logits"])
@pytest.mark.parametrize("n,V,dtype", [(129, 40001, F32), (131, 70003, BF16)], ids=["f32", "bf16"])
def test_batches_of_long_rows(gpu_lib, n, V, dtype, kind):
    """More rows than have two work-groups each, longer than one's registers hold."""
    print(f"[case] sample batch of long rows {n} {V} {dtype} {kind}", flush=True)
    g = torch.Generator().manual_seed(V)
    x, u = _logits(n, V, dtype, seed=n)
    x[5::9, V // 3:] = -float("inf")
    kw = dict(temperature=torch.rand(n, generator=g) + 0.4, top_p=torch.rand(n, generator=g) * 0.8 + 0.1,
              top_k=torch.randint(0, 900, (n,), generator=g, dtype=torch.int32), min_p=torch.rand(n, generator=g) * 0.02)
    kw["top_k"][::2] = 0                       # by top-p alone
    kw["top_p"][1::4] = 1.0                    # by top-k alone
    kw["top_k"][8::8] = 1500                   # and by top-p behind a long top-k
    kw = {k: v.cuda() for k, v in kw.items()}
    tokens, out = _run(x, u, kind, **kw)
    rows = dict(probs=out if kind == "probs" else None, kept=out if kind == "kept_logits" else None)
    _check(x, u, tokens, *(kw[k] for k in ("temperature", "top_k", "top_p", "min_p")), **rows)
    _holds(x, tokens, kw["temperature"], **rows)
    if kind:                                   # and in place
        y, again = x.clone(), torch.empty_like(tokens)
        Sampler().run(y, u, again, **{kind: y}, **kw)
        torch.cuda.synchronize()
        assert torch.equal(y, out) and torch.equal(again, tokens)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [32000, 128256])
@pytest.mark.parametrize("first", [0, 13, 20000])
def test_unmasked_tokens_beside_each_other(gpu_lib, first, V, dtype):
    """3000 neighbouring ids are left by a mask: few threads have them all."""
    print(f"[case] sample neighbours {first} {V} {dtype}", flush=True)
    x, u = _logits(5, V, dtype, seed=first + 1)
    x[:, :first] = -float("inf")
    x[:, first + 3000:] = -float("inf")
    for kw in (dict(top_k=_i(257, 400, 511, 512, 3)), dict(top_k=_i(400, 376, 375, 374, 2999), top_p=_f(0.9, 0.5, 0.99, 1.0, 0.8)),
               dict(top_k=_i(513, 1024, 1025, 2900, 3000), top_p=_f(0.9, 0.5, 0.99, 1.0, 0.8))):
        tokens, out = _run(x, u, "probs", **kw)
        _check(x, u, tokens, None, kw["top_k"], kw.get("top_p"), probs=out)
        _holds(x, tokens, probs=out)
