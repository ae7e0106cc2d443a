"""GPU: appended, committed and copied rows of a captured graph, K and V, every
place that they write."""
import pytest
import torch

from cache_util import BF16, Paged
from paper_2505_17074_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spare", [5, (1 << 32) // (64 * 2 * 128 * 2) + 100], ids=["small", "past_4_gib"])
def test_replays_write_what_eager_calls_write(gpu_lib, spare):
    print(f"[case] movers replayed, {spare} spare pages", flush=True)
    par = [-1, 0, 0, 1, 1, 2, 2, 3, 3, 4, 4, 5, 5, 6, 6]
    p = Paged([70, 5], [15, 15], 2, 128, spare=spare, far=True, seed=3, fill=0.0)
    p.write(p.ctx)
    k_new, v_new = p.new_rows()
    chunks, req = p.chunks(), B.make_requests([70, 5], None, par)
    node = torch.tensor([13, 9], dtype=torch.int32, device="cuda")
    used = sorted(set(p.table_np[0, :2].tolist() + p.table_np[1, :1].tolist()))
    copies = [[used[0], 3, 64], [used[1], 1, 11]]
    look = used + [1, 3]
    start = p.k[:, look].clone(), p.v[:, look].clone()

    def reset():
        p.k[:, look], p.v[:, look] = start

    def call():
        p.cache.append(chunks, k_new, v_new)
        p.cache.commit(req, node)
        p.cache.copy_pages(copies)

    call()
    torch.cuda.synchronize()
    want = p.k[:, look].clone(), p.v[:, look].clone()
    for w, s, new in zip(want, start, (k_new, v_new)):
        assert not torch.equal(w, s)
        assert torch.equal(w[:, -1], w[:, 0]) and torch.equal(w[:, -2, :11], w[:, 1, :11])       # the copies
        at = [used.index(int(x)) for x in p.where(0, [70, 71, 72, 73])[0]]
        path = [0, 2, 6, 13]                                                                     # of the accepted node
        for t, x in enumerate(path):
            assert torch.equal(w[0, at[t], (70 + t) % 64], new[0, x])
    reset()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for other in range(4):
        reset()
        if other % 2:                                    # eager work of the same kind between the replays
            p.cache.append(chunks, k_new, v_new)
            torch.cuda.synchronize()
            reset()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.k[:, look], want[0]) and torch.equal(p.v[:, look], want[1]), other
    del p, want, start, g
    torch.cuda.empty_cache()
