"""GPU: ChunkAttention refuses to be captured, on the capturing stream by name
and as the current one, and works before, beside and after."""
import pytest
import torch

from cache_util import BF16, Paged, queries
from paper_2505_17074_amd.cache import ChunkAttention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("named", [False, True], ids=["current", "named"])
def test_a_captured_call_is_refused(gpu_lib, named):
    print(f"[case] chunk capture refused {named}", flush=True)
    p = Paged([900, 3], [2, 70], 2, 128, seed=4).write()
    q = queries(72, 8, 128, seed=4).cuda()
    ref, out = (torch.zeros((72, 8, 128), dtype=BF16, device="cuda") for _ in range(2))
    att = ChunkAttention(p.cache, 8)
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    att.run(p.chunks(), q, ref, stream=stream)           # nothing left to grow, and the stream is known
    torch.cuda.synchronize()
    x = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    before = att._i
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream, capture_error_mode="relaxed"):
        x.add_(1)
        with pytest.raises(RuntimeError, match="staging of their own"):
            if named:
                with torch.cuda.stream(other):
                    att.run(p.chunks(), q, out, stream=stream)
            else:
                att.run(p.chunks(), q, out)
        x.add_(1)
    assert att._i == before                              # no slot was taken
    for _ in range(2):
        g.replay()
        att.run(p.chunks(), q, out, stream=other)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
        out.zero_()
    assert (x == 4).all()


def test_an_object_that_ends_inside_a_capture(gpu_lib):
    """Its buffers stay until the capture is over, and not for good."""
    import gc
    from paper_2505_17074_amd import cache as module
    print("[case] chunk object ends in a capture", flush=True)
    gc.collect()
    p = Paged([900], [2], 2, 128, seed=5).write()
    q = queries(2, 8, 128, seed=5).cuda()
    out, ref = (torch.zeros((2, 8, 128), dtype=BF16, device="cuda") for _ in range(2))
    ChunkAttention(p.cache, 8).run(p.chunks(), q, ref)
    assert not module._kept
    x = torch.zeros(4, device="cuda")
    att = ChunkAttention(p.cache, 8)
    att.run(p.chunks(), q, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, capture_error_mode="relaxed"):
        x.add_(1)
        ws = att._ws.data_ptr()
        del att
        assert [w.data_ptr() for _, w, _ in module._kept] == [ws]
    g.replay()
    again = ChunkAttention(p.cache, 8)
    assert not module._kept
    again.run(p.chunks(), q, out)
    torch.cuda.synchronize()
    assert torch.equal(out, ref) and (x == 1).all()
