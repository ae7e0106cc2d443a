"""GPU: block tables and pools that are let go while calls on another stream
still read them."""
import numpy as np
import pytest
import torch

from cache_util import BF16, Paged, queries
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention, PagedCache

pytestmark = pytest.mark.gpu


def _busy(stream):
    """Work that a call on the stream waits behind (a few milliseconds)."""
    a = torch.ones((4096, 4096), device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(8):
            a = torch.mm(a, a).clamp_(max=1)
    return a


@pytest.mark.parametrize("named", [True, False], ids=["named", "current"])
@pytest.mark.parametrize("what", ["append", "commit", "attention"])
def test_a_replaced_table_stays_until_its_calls_have_ended(gpu_lib, what, named):
    """Whoever takes a dropped table's memory fills it with another request's
    page ids; the call that was given the old one still goes by them."""
    print(f"[case] replaced table {what} {named}", flush=True)
    p = Paged([40, 70], [6, 15], 2, 128, 32, seed=8, fill=0.0).write()
    k_new, v_new = (x + 1 for x in p.new_rows())
    q = queries(21, 8, 128, seed=8).cuda()
    tree = B.make_requests([40, 70], tree_parents=[[-1, 0, 0, 2, 3, 4], [-1] + [i // 2 for i in range(14)]])
    node = torch.tensor([5, 11], dtype=torch.int32, device="cuda")
    outs = [torch.empty((21, 8, 128), dtype=BF16, device="cuda") for _ in range(2)]
    att, side, start = ChunkAttention(p.cache, 8), torch.cuda.Stream(), (p.k.clone(), p.v.clone())

    def call(out, stream=None):
        if what == "append":
            p.cache.append(p.chunks(), k_new, v_new, stream=stream)
        elif what == "commit":
            p.cache.commit(tree, node, stream=stream)
        else:
            att.run(p.chunks(), q, out, stream=stream)

    call(outs[0])
    torch.cuda.synchronize()
    want = p.k.clone(), p.v.clone()
    p.k.copy_(start[0])
    p.v.copy_(start[1])
    shape = p.table.shape
    p.cache.table = None
    p.table = p.table.clone()              # the only references to the table from here on: these two
    for _ in range(3):
        p.cache.table = p.table
        torch.cuda.synchronize()
        keep = _busy(side)
        if named:
            call(outs[1], side)
        else:
            with torch.cuda.stream(side):
                call(outs[1])
        p.cache.table = p.table = None
        others = [torch.zeros(shape, dtype=torch.int32, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        assert torch.equal(p.k, want[0]) and torch.equal(p.v, want[1]) and (what != "attention" or torch.equal(outs[0], outs[1]))
        p.k.copy_(start[0])
        p.v.copy_(start[1])
        outs[1].zero_()
        p.table = torch.from_numpy(np.ascontiguousarray(p.table_np)).cuda()
        del keep, others


def test_pools_that_end_with_work_pending(gpu_lib):
    print("[case] pools let go", flush=True)
    side = torch.cuda.Stream()
    q, chunks = queries(9, 8, 128, seed=1).cuda(), B.make_chunks([2000], [9])
    att = None
    for _ in range(4):
        k, v = (torch.ones((1, 300, 32, 2, 128), dtype=BF16, device="cuda") for _ in range(2))
        out = torch.zeros((9, 8, 128), dtype=BF16, device="cuda")
        c = PagedCache(k, v, torch.arange(300, dtype=torch.int32, device="cuda")[None])
        if att is None:
            att = ChunkAttention(c, 8)
            att.run(chunks, q, out)                      # nothing left to grow
        att.cache = c
        torch.cuda.synchronize()
        keep = _busy(side)
        att.run(chunks, q, out, stream=side)
        shape = k.shape
        att.cache = None
        del c, k, v
        others = [torch.full(shape, 3.0, dtype=BF16, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert (out == 1).all()
        del keep, others
