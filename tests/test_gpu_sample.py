"""GPU: sampled tokens and their distributions against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.sample import Sampler

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# Weights are off by 1e-11 of their value.  Sums in fixed point are off by a unit a
# term at most: a list's by n 2^-48, histograms' by n 2^-50 or, for the 62 bits of
# the sum of n weights, by n (2 n) 2^-62, of the largest weight, and less of the
# total.  A border is a share of such a sum and is compared with another: twice that.
def near_of(n):
    return 2 * (1e-11 + n * 2.0 ** -48 + n * n * 2.0 ** -61)


# Probabilities: a weight over a sum in 64 bits (a list's weights in units of 2^-48).
PROB = 4e-10


def _check(logits, u, tokens, T=None, k=None, p=None, m=None, probs=None, kept=None, whole=False, flat=False):
    """whole: all weights are 1, so that every sum, and its product with an fp32 share
    (24 + 15 bits), is exact in 64 bits: nothing is too near to a border.  flat:
    single tokens may weigh less than the distance that sums of so many are off by
    (3e6 of 3e-7 each, where that is 1.8e-5); what such rows hold is a distribution
    and one of its tokens."""
    x = logits.double().cpu().numpy()
    row = lambda t, i, z: z if t is None else t[i].item()  # noqa: E731
    near = 0
    for i in range(x.shape[0]):
        temp = row(T, i, 1.0)
        token, q, ids, margin = oracle.sample(x[i], u[i].item(), temp, row(k, i, 0), row(p, i, 1.0), row(m, i, 0.0))
        if margin <= near_of(x.shape[1]) and not whole:
            near += 1
            if flat:
                got = probs[i].double().cpu().numpy()
                # each probability is rounded by half a step of its own
                assert abs(got.sum() - 1) <= 2.0 ** -8 + PROB and got[tokens[i].item()] > 0
            continue
        assert tokens is None or tokens[i].item() == token, (i, tokens[i].item(), token, margin)
        half = 2.0 ** -8 if logits.dtype == BF16 else 2.0 ** -24
        if probs is not None:
            got = probs[i].double().cpu().numpy()
            assert (np.abs(got - q) <= q * (half * 1.001 + PROB) + 2.0 ** -126).all(), i
        if kept is not None:
            got = kept[i].double().cpu().numpy()
            stays = np.zeros(x.shape[1], bool)
            stays[ids] = True
            assert (got[~stays] == torch.finfo(logits.dtype).min).all(), i
            one = not temp > 0 or not row(p, i, 1.0) > 0 or not row(m, i, 0.0) <= 1
            want = np.zeros(len(ids)) if one else x[i][ids] / temp
            assert (np.abs(got[ids] - want) <= np.abs(want) * half * 1.001 + 2.0 ** -126).all(), i
    assert near * 10 <= x.shape[0] or near <= 1 or flat


def _run(logits, u, kind=None, **kw):
    n = logits.shape[0]
    tokens = torch.full((n + 2,), -9, dtype=torch.int32, device="cuda")
    out = None
    if kind:
        out = torch.full_like(logits, float("nan"))
        kw[kind] = out
    Sampler().run(logits, u, tokens[:n], **kw)
    torch.cuda.synchronize()
    assert (tokens[n:] == -9).all()
    return tokens[:n], out


def _logits(n, V, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, V), generator=g) * spread
    x[:, torch.randint(0, V, (max(1, V // 200),), generator=g)] += 5.0
    return x.to(dtype).cuda(), torch.rand(n, generator=g).cuda()


def _f(*x):
    return torch.tensor(x, dtype=F32, device="cuda")


def _i(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


FILTERS = {
    "none": {},
    "temperature": dict(temperature=[0.3, 1.0, 1.7, 0.0, 5.0]),
    "top_k": dict(top_k=[1, 5, 50, 0, 700]),
    "top_p": dict(top_p=[0.1, 0.9, 0.5, 1.0, 0.999]),
    "min_p": dict(min_p=[0.01, 0.5, 0.0, 1.0, 1e-6]),
    "all": dict(temperature=[0.3, 1.0, 1.7, 0.0, 0.8], top_k=[1, 50, 2000, 0, 300], top_p=[0.9, 0.95, 0.5, 0.4, 0.99],
                min_p=[0.0, 0.02, 0.1, 0.05, 0.001]),
}


def _filters(name):
    return {k: (_i if k == "top_k" else _f)(*v) for k, v in FILTERS[name].items()}


@pytest.mark.parametrize("kind", [None, "probs", "kept_logits"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 1000, 4099, 32000, 50257, 128256])
@pytest.mark.parametrize("name", FILTERS)
def test_matches_the_oracle(gpu_lib, name, V, dtype, kind):
    print(f"[case] sample {name} {V} {dtype} {kind}", flush=True)
    kw = _filters(name)
    x, u = _logits(5, V, dtype, seed=V + len(name))
    tokens, out = _run(x, u, kind, **kw)
    _check(x, u, tokens, *(kw.get(k) for k in ("temperature", "top_k", "top_p", "min_p")),
           probs=out if kind == "probs" else None, kept=out if kind == "kept_logits" else None)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("what", ["one_value", "two_values", "few_values", "two_values_high"])
def test_equal_logits(gpu_lib, what, dtype):
    """Runs of equal logits longer than any list, cut among the ids."""
    V = 30011
    print(f"[case] sample ties {what} {dtype}", flush=True)
    g = torch.Generator().manual_seed(3)
    x = {"one_value": torch.full((5, V), -3.25),
         "two_values": (torch.rand((5, V), generator=g) < 0.9).float() * -1.0,
         "few_values": torch.randint(0, 5, (5, V), generator=g).float() * 0.25,
         "two_values_high": (torch.rand((5, V), generator=g) < 0.001).float() * 4.0}[what].to(dtype).cuda()
    u = torch.rand(5, generator=g).cuda()
    for kw in (dict(top_k=_i(1, 2, 5000, 29000, 30010)), dict(top_p=_f(0.1, 0.5, 0.75, 0.9, 0.999)),
               dict(top_k=_i(0, 20000, 5000, 29000, 1025), top_p=_f(0.1, 0.5, 0.75, 0.9, 0.3)),
               dict(min_p=_f(0.1, 0.5, 1.0, 0.9, 0.0))):
        tokens, out = _run(x, u, "probs", **kw)
        _check(x, u, tokens, None, kw.get("top_k"), kw.get("top_p"), kw.get("min_p"), probs=out, whole=what == "one_value")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_masked_and_not_finite(gpu_lib, dtype):
    V = 5003
    print(f"[case] sample masked {dtype}", flush=True)
    x, u = _logits(8, V, dtype, seed=9)
    low = torch.finfo(dtype).min
    x[0] = -float("inf")
    x[1] = float("nan")
    x[2, 100:] = low
    x[3, :4990] = -float("inf")
    x[4, ::2] = float("nan")
    x[5, 7] = x[5, 4000] = float("inf")
    x[6] = low
    x[7, 1:] = -float("inf")
    kws = (dict(), dict(top_k=_i(*[300] * 8)), dict(top_p=_f(*[0.9] * 8)), dict(temperature=_f(*[0.5] * 8), min_p=_f(*[0.01] * 8)),
           dict(temperature=_f(*[0.0] * 8)), dict(top_k=_i(*[5000] * 8), top_p=_f(*[0.99] * 8)))
    for kw in kws:
        tokens, out = _run(x, u, "probs", **kw)
        assert tokens[:2].tolist() == [-1, -1] and (out[:2] == 0).all()
        _check(x, u, tokens, *(kw.get(k) for k in ("temperature", "top_k", "top_p", "min_p")), probs=out)
    tokens, out = _run(x, u, "kept_logits", top_k=_i(*[3] * 8))
    assert (out[:2] == low).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [3000, 40000])
def test_zeros_of_both_signs(gpu_lib, V, dtype):
    """They are equal, so the lower id comes first."""
    print(f"[case] sample signed zeros {V} {dtype}", flush=True)
    x = torch.full((6, V), -1.0)
    x[:, 1::7] = 0.0
    x[:, 4::7] = -0.0
    x = x.to(dtype).cuda()
    u = _f(0.0, 0.2, 0.4, 0.6, 0.8, 0.99)
    for kw in (dict(top_k=_i(1, 2, 3, 50, 300, 512)), dict(top_p=_f(1e-4, 1e-3, 0.01, 0.1, 0.3, 0.45)),
               dict(top_k=_i(*[2] * 6), temperature=_f(*[0.0] * 6)), dict(top_k=_i(600, 601, 700, 800, 513, 514))):
        tokens, out = _run(x, u, "probs", **kw)
        _check(x, u, tokens, *(kw.get(k) for k in ("temperature", "top_k", "top_p", "min_p")), probs=out)


def test_extreme_parameters(gpu_lib):
    print("[case] sample extremes", flush=True)
    nan, inf = float("nan"), float("inf")
    x, _ = _logits(12, 1500, F32, seed=4)
    u = _f(0.0, 0.5, 1 - 2.0 ** -24, 0.3, 0.0, 0.999, 0.1, 0.2, 0.3, 0.4, 0.5, 0.6)
    first = x.argmax(-1).tolist()
    def run(**kw):
        tokens, out = _run(x, u, "probs", **kw)
        _check(x, u, tokens, *(kw.get(k) for k in ("temperature", "top_k", "top_p", "min_p")), probs=out)
        return tokens.tolist()
    assert run(temperature=_f(*[0.0, -1.0, nan, -inf] * 3)) == first
    assert run(top_p=_f(*[0.0, -1.0, nan, -inf] * 3)) == first
    assert run(min_p=_f(*[1.5, inf, nan, 2.0] * 3)) == first
    assert run(top_k=_i(*[1] * 12)) == first
    assert run(temperature=_f(*[1e-30, 1e-38, 1e-45, 1e-6] * 3)) == first
    run(temperature=_f(*[inf, 1e30, 1e6, 3e38] * 3))
    run(temperature=_f(*[inf, 1e30, 1e6, 3e38] * 3), top_k=_i(*[100] * 12), top_p=_f(*[0.3] * 12))
    run(top_k=_i(*[-5, 0, 1500, 1501, 2**31 - 1, 1499] * 2), top_p=_f(*[1.0, 2.0, inf, 1 - 2.0 ** -24] * 3),
        min_p=_f(*[0.0, -1.0, -inf, 1e-30] * 3))
    run(temperature=_f(*[0.02] * 12), top_k=_i(*[1400] * 12))               # what stays has weights of zero


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("spread", [1e-3, 30.0, 1e30])
def test_narrow_and_wide_logits(gpu_lib, spread, dtype):
    print(f"[case] sample spread {spread} {dtype}", flush=True)
    x, u = _logits(5, 20011, dtype, seed=6, spread=spread)
    for kw in (dict(top_k=_i(3, 100, 5000, 15000, 20000)), dict(top_p=_f(0.2, 0.5, 0.9, 0.99, 0.01)), {}):
        tokens, out = _run(x, u, "probs", **kw)
        _check(x, u, tokens, None, kw.get("top_k"), kw.get("top_p"), probs=out)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("start", [0, 1, 3, 6])
def test_strides_and_alignment(gpu_lib, start, dtype):
    """Rows that begin anywhere, in a wider array; outputs that begin elsewhere."""
    print(f"[case] sample strides {start} {dtype}", flush=True)
    V = 4001
    x, u = _logits(5, V, dtype, seed=7)
    wide = torch.full((5, V + 13), 50.0, dtype=dtype, device="cuda")
    wide[:, start:start + V] = x
    kw = _filters("all")
    for shift in (start, start + 1):
        out = torch.full((5, V + 21), 7.0, dtype=dtype, device="cuda")
        tokens = torch.empty(5, dtype=torch.int32, device="cuda")
        Sampler().run(wide[:, start:start + V], u, tokens, probs=out[:, shift:shift + V], **kw)
        torch.cuda.synchronize()
        _check(x, u, tokens, *(kw[k] for k in ("temperature", "top_k", "top_p", "min_p")), probs=out[:, shift:shift + V])
        assert (out[:, :shift] == 7.0).all() and (out[:, shift + V:] == 7.0).all()
    assert (wide[:, :start] == 50.0).all() and torch.equal(wide[:, start:start + V], x)


@pytest.mark.parametrize("kind", ["probs", "kept_logits"])
@pytest.mark.parametrize("V", [999, 128257])
def test_in_place(gpu_lib, kind, V):
    print(f"[case] sample in place {kind} {V}", flush=True)
    kw = _filters("all")
    x, u = _logits(5, V, BF16, seed=8)
    tokens, out = _run(x, u, kind, **kw)
    y = x.clone()
    again = torch.empty(5, dtype=torch.int32, device="cuda")
    Sampler().run(y, u, again, **{kind: y}, **kw)
    torch.cuda.synchronize()
    assert torch.equal(y, out) and torch.equal(again, tokens)
    none = torch.full_like(x, float("nan"))
    Sampler().run(x, **{kind: none}, **kw)                                  # the rows alone
    torch.cuda.synchronize()
    assert torch.equal(none, out)


@pytest.mark.parametrize("V,dtype", [(700001, F32), (1100003, BF16), (4500001, BF16)], ids=["f32", "bf16", "bf16_longer"])
def test_very_long_rows(gpu_lib, V, dtype):
    """Runs of ids of several loads, more of them a thread than it has bits for."""
    print(f"[case] sample long {V} {dtype}", flush=True)
    x, u = _logits(2, V, dtype, seed=V, spread=6.0)
    x[:, V - 5] = 50.0 if dtype == BF16 else 30.0          # past the bf16 table, near the row's end
    x[:, :V // 3] = -float("inf")
    for kw in (dict(), dict(top_p=_f(0.9, 0.6), temperature=_f(1.0, 6.0)), dict(top_k=_i(50, 2000)),
               dict(top_p=_f(0.99, 0.2), temperature=_f(8.0, 8.0))):
        tokens, out = _run(x, u, "probs", **kw)
        _check(x, u, tokens, *(kw.get(k) for k in ("temperature", "top_k", "top_p", "min_p")), probs=out,
               flat=V > 1 << 22 and "temperature" in kw)


def test_frequencies(gpu_lib):
    """Uniforms on a grid: each token comes up as often as its probability says."""
    print("[case] sample frequencies", flush=True)
    n = 4096
    x = torch.log(torch.tensor([0.5, 0.05, 0.2, 0.15, 0.1])).repeat(n, 1).cuda()
    u = (torch.arange(n, device="cuda", dtype=F32) + 0.5) / n
    tokens, _ = _run(x, u, top_k=torch.full((n,), 4, dtype=torch.int32, device="cuda"))
    got = torch.bincount(tokens.long(), minlength=5).double().cpu() / n
    assert (got - torch.tensor([0.5, 0, 0.2, 0.15, 0.1]).double() / 0.95).abs().max() <= 1.0 / n


@pytest.mark.parametrize("n,V", [(5, 32000), (1, 128256), (300, 1000)])
def test_replayed_and_on_other_streams(gpu_lib, n, V):
    print(f"[case] sample replay {n} {V}", flush=True)
    kw = {k: v.repeat(n // 5 + 1)[1:n + 1].contiguous() for k, v in _filters("all").items()}
    x, u = _logits(n, V, F32, seed=11)
    s = Sampler()
    tokens, out = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty_like(x)
    a = B.SpecSampleArgs()
    a.num_rows, a.vocab, a.dtype, a.rows_kind = n, V, B.SPEC_F32, B.SPEC_SAMPLE_PROBS
    a.logits, a.uniforms, a.tokens, a.rows = (t.data_ptr() for t in (x, u, tokens, out))
    a.logits_stride = a.rows_stride = V
    a.temperature, a.top_k, a.top_p, a.min_p = (kw[k].data_ptr() for k in ("temperature", "top_k", "top_p", "min_p"))
    st, need = B.spec_sample_workspace_bytes(a)
    assert st == B.SPEC_OK
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")           # it may hold anything
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        B.check(B.spec_sample(a, (ws.data_ptr() + 255) // 256 * 256, need, stream.cuda_stream), "spec_sample")
        with pytest.raises(RuntimeError):
            s.run(x, u, tokens, probs=out, stream=stream, **kw)
    for i in range(4):
        y, v = _logits(n, V, F32, seed=20 + i)
        x.copy_(y)
        u.copy_(v)
        tokens.fill_(-3)
        torch.cuda.synchronize()
        graph.replay()
        again, rows = torch.empty_like(tokens), torch.empty_like(out)
        torch.cuda.synchronize()
        s.run(x, u, again, probs=rows, stream=torch.cuda.Stream() if i % 2 else None, **kw)
        torch.cuda.synchronize()
        assert torch.equal(again, tokens) and torch.equal(rows, out)
        _check(x, u, tokens, *(kw[k] for k in ("temperature", "top_k", "top_p", "min_p")), probs=out)


def test_growing_batches(gpu_lib):
    """One object: batches that need more workspace, on streams in turn."""
    print("[case] sample growing", flush=True)
    s, streams = Sampler(), [torch.cuda.Stream() for _ in range(3)]
    jobs = []
    for i, (n, V) in enumerate([(1, 100), (3, 5000), (2, 128256), (64, 32000), (1, 100), (200, 9000)]):
        x, u = _logits(n, V, BF16 if i % 2 else F32, seed=i)
        p, tokens = torch.full((n,), 0.8, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        jobs.append((x, u, p, tokens))
    torch.cuda.synchronize()
    for i, (x, u, p, tokens) in enumerate(jobs):
        s.run(x, u, tokens, top_p=p, stream=streams[i % 3])
    torch.cuda.synchronize()
    for x, u, p, tokens in jobs:
        _check(x, u, tokens, p=p)


def test_many_rows(gpu_lib):
    print("[case] sample many rows", flush=True)
    n = 300
    g = torch.Generator().manual_seed(2)
    x, u = _logits(n, 3001, F32, seed=12)
    kw = dict(temperature=(torch.rand(n, generator=g) + 0.3).cuda(), top_k=torch.randint(0, 600, (n,), generator=g, dtype=torch.int32).cuda(),
              top_p=(torch.rand(n, generator=g) * 0.9 + 0.1).cuda(), min_p=(torch.rand(n, generator=g) * 0.05).cuda())
    tokens, out = _run(x, u, "probs", **kw)
    _check(x, u, tokens, *(kw[k] for k in ("temperature", "top_k", "top_p", "min_p")), probs=out)


def test_drafts_and_their_acceptance(gpu_lib):
    """A draft's tokens and rows, a target's truncated rows, and the acceptance
    test that reads them: the next tokens are the target distribution's own."""
    print("[case] sample and accept", flush=True)
    n, V = 6, 1000
    nq = 3 * n
    target, _ = _logits(nq, V, F32, seed=13)
    draft, u = _logits(2 * n, V, F32, seed=14)
    s = Sampler()
    tokens, q = torch.empty(2 * n, dtype=torch.int32, device="cuda"), torch.empty_like(draft)
    s.run(draft, u, tokens, temperature=torch.full((2 * n,), 0.8, device="cuda"),
          top_k=torch.full((2 * n,), 20, dtype=torch.int32, device="cuda"), probs=q)
    kept = torch.empty_like(target)
    T, p = torch.full((nq,), 0.7, device="cuda"), torch.full((nq,), 0.9, device="cuda")
    s.run(target, temperature=T, top_p=p, kept_logits=kept)
    uniforms = torch.rand(nq, generator=torch.Generator().manual_seed(5)).cuda()
    req = B.make_requests([5] * n, [2] * n)
    a = B.SpecAcceptArgs()
    a.vocab, a.dtype = V, B.SPEC_F32
    a.target_logits, a.logits_stride, a.draft_probs, a.probs_stride = kept.data_ptr(), V, q.data_ptr(), V
    length, token = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
    a.draft_tokens, a.uniforms, a.accepted_len, a.next_token = (t.data_ptr() for t in (tokens, uniforms, length, token))
    st, dev, host = B.spec_workspace_bytes(req, None, a)
    assert st == B.SPEC_OK
    ws = torch.empty(dev + 256, dtype=torch.uint8, device="cuda")
    staging = torch.empty(max(host, 1), dtype=torch.uint8, pin_memory=True)
    stream = torch.cuda.current_stream()
    B.check(B.spec_accept(req, a, (ws.data_ptr() + 255) // 256 * 256, dev, staging.data_ptr(), host, stream.cuda_stream), "accept")
    torch.cuda.synchronize()
    x = target.double().cpu().numpy()
    rows = np.stack([oracle.sample(x[i], 0.5, T[i].item(), 0, p[i].item())[1] for i in range(nq)])
    for i in range(n):
        here, got = 0, tokens[2 * i:2 * i + 2].tolist()
        q64 = q[2 * i:2 * i + 2].double().cpu().numpy()
        while here < 2 and uniforms[3 * i + here].item() * q64[here][got[here]] < rows[3 * i + here][got[here]]:
            here += 1
        assert length[i].item() == here
        left = rows[3 * i + here] if here == 2 else np.maximum(rows[3 * i + here] - q64[here], 0)
        assert token[i].item() == _first(left, uniforms[3 * i + 2].item())


def _first(w, u):
    total = np.cumsum(w)
    return int(np.searchsorted(total, u * total[-1], side="right"))
