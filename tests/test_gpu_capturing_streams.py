"""GPU: objects used on another stream while the stream of their last call
captures a graph: refused, the graph is what it would have been, and the next
call after the capture works."""
import pytest
import torch

from cache_util import BF16, Paged, queries
from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import ChunkAttention
from paper_2505_17074_amd.sample import Sampler

pytestmark = pytest.mark.gpu


def test_a_sampler(gpu_lib):
    print("[case] sample beside a capture", flush=True)
    s = Sampler()
    x, u = torch.randn((3, 5000), device="cuda"), torch.rand(3, device="cuda")
    tokens, again = (torch.full((3,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    s.run(x, u, tokens, stream=stream)
    torch.cuda.synchronize()
    y = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream, capture_error_mode="relaxed"):
        y.add_(1)
        with pytest.raises(RuntimeError, match="captur"):
            s.run(x, u, again, stream=other)
        y.add_(1)
    for i in range(1, 4):
        g.replay()
        s.run(x, u, again, stream=other)
        torch.cuda.synchronize()
        assert torch.equal(again, tokens) and (y == 2 * i).all()
        again.fill_(-9)


@pytest.mark.parametrize("kind", ["plain", "window", "prefixes"])
def test_an_attention(gpu_lib, kind):
    print(f"[case] attention beside a capture {kind}", flush=True)
    p = Paged([900, 900], [2, 1], 2, 128, seed=4).write()
    q = queries(3, 8, 128, seed=4).cuda()
    ref, out = (torch.zeros((3, 8, 128), dtype=BF16, device="cuda") for _ in range(2))
    att = ChunkAttention(p.cache, 8, window=200 if kind == "window" else None)
    kw = dict(prefixes=B.make_prefixes([2], [0])) if kind == "prefixes" else {}
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    att.run(p.chunks(), q, ref, stream=stream, **kw)
    torch.cuda.synchronize()
    y = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    before = att._i
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream, capture_error_mode="relaxed"):
        y.add_(1)
        with pytest.raises(RuntimeError, match="would take this call in"):
            att.run(p.chunks(), q, out, stream=other, **kw)
        y.add_(1)
    assert att._i == before
    for i in range(1, 4):
        g.replay()
        att.run(p.chunks(), q, out, stream=other, **kw)
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and (y == 2 * i).all()
        out.zero_()
