"""GPU: rotated rows of whole prompts: many rows a call, and so many bytes that
they are stored past the caches.  Every row is what a call of few rows makes of
it, bit for bit, and some are checked against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from cache_util import BF16, F32, Paged
from paper_2505_17074_amd import binding as B
from test_gpu_rotate import _check, _freq, _rows, turned

pytestmark = pytest.mark.gpu

CASES = {
    # name: ctx, new, query heads, KV heads, d, page tokens, rotated elements, dtype
    "many_rows": ([0, 37, 1000, 3, 64], [1501, 7, 2002, 63, 650], 4, 2, 64, 64, 64, BF16),
    "many_rows_f32": ([5, 0, 31], [1502, 2001, 801], 5, 1, 96, 32, 64, F32),
    "one_prompt": ([7], [4099], 3, 3, 128, 96, 128, BF16),
    "many_bytes": ([0, 100, 31, 7], [4001, 3, 3600, 3400], 32, 8, 128, 64, 128, BF16),      # 135 MB read and written
    "many_bytes_f32": ([9, 2], [4321, 1211], 32, 8, 128, 64, 128, F32),
}


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("name", CASES)
def test_prompts(gpu_lib, name, interleaved):
    ctx, new, hq, hkv, d, page, rotary, dtype = CASES[name]
    print(f"[case] rotate prompts {name} {interleaved}", flush=True)
    n = sum(new)
    p = Paged(ctx, new, hkv, d, page, dtype=dtype, seed=len(name))
    k, v = (x[0] for x in p.new_rows())
    q = torch.randn((n, hq, d), generator=torch.Generator("cuda").manual_seed(3), device="cuda").to(dtype)
    q_out, want = torch.full((n + 2, hq, d), 7.0, dtype=dtype, device="cuda"), torch.empty_like(q)
    freq = _freq(rotary)
    p.cache.append_rotated(p.chunks(), k, v, freq.cuda(), q, q_out, interleaved=interleaved)
    torch.cuda.synchronize()
    assert (q_out[n:] == 7.0).all()
    got = [x.clone() for x in _rows(p)]                    # everything else is NaN still

    # the same in calls of up to 500 rows
    p.k.fill_(float("nan"))
    p.v.fill_(float("nan"))
    left, at, first = list(new), list(ctx), np.cumsum([0] + list(new))
    while any(left):
        step = [min(x, 500) if i == next(j for j, y in enumerate(left) if y) else 0 for i, x in enumerate(left)]
        i = next(j for j, y in enumerate(step) if y)
        r0 = first[i] + new[i] - left[i]
        part = slice(int(r0), int(r0) + step[i])
        p.cache.append_rotated(B.make_chunks(at, step), k[part], v[part], freq.cuda(), q[part], want[part],
                               interleaved=interleaved)
        at[i] += step[i]
        left[i] -= step[i]
    torch.cuda.synchronize()
    assert torch.equal(q_out[:n], want)
    assert all(torch.equal(x, y) for x, y in zip(got, _rows(p))) and torch.equal(got[1], v)

    pick = np.random.default_rng(1).choice(n, 60, replace=False)
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(ctx, new)])[pick]
    pick = torch.from_numpy(pick).cuda()
    _check(q_out[pick], *turned(q[pick], pos, freq, interleaved, dtype))
    _check(got[0][pick], *turned(k[pick], pos, freq, interleaved, dtype))
