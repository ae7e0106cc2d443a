"""GPU: how precisely a bf16 output of the chunk attention is computed before
its own rounding."""
import copy

import numpy as np
import pytest
import torch

from cache_util import BF16, U32, Paged, queries, reference
from paper_2505_17074_amd.cache import ChunkAttention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ctx,new,hq,hkv,d", [
    ([0, 1, 31, 64, 700, 2500], [1] * 6, 8, 2, 128), ([1000], [1], 32, 8, 128), ([5000, 40], [8, 3], 8, 2, 128),
    ([300, 900, 0], [32, 5, 20], 2, 2, 64), ([2111, 7], [1, 1], 16, 4, 64)])
def test_few_rows_lose_nothing_before_the_outputs_rounding(gpu_lib, ctx, new, hq, hkv, d):
    """At most 32 query rows a KV head: weights in two bf16 parts, each half a
    step (2^-8) of what is left, so 2^-16 of a weight at most; the fp32 sums as
    in `reference`; then one rounding to bf16, half a step of what was computed."""
    print(f"[case] chunk bf16 precision {ctx} {new} {hq}/{hkv} d {d}", flush=True)
    p = Paged(ctx, new, hkv, d, 64, seed=sum(new) + d).write()
    q = queries(sum(new), hq, d, seed=3)
    out = torch.empty((sum(new), hq, d), dtype=BF16, device="cuda")
    ChunkAttention(p.cache, hq).run(p.chunks(), q.cuda(), out)
    ref, bound = reference(p, q, out=torch.float32)      # sums, exponents, U32 of the result
    positive = copy.copy(p)
    positive.rows = [(k, v.abs()) for k, v in p.rows]
    size, _ = reference(positive, q, out=torch.float32)  # sum of weight times |v|
    before = bound + 2.0 ** -16 * size
    off = np.abs(out.double().cpu().numpy() - ref) / (before + 2.0 ** -8 * (np.abs(ref) + before))
    assert off.max() <= 1.0, off.max()
