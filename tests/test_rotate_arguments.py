"""What the rotated append refuses, on a host without a GPU: the checks run
before the first HIP call."""
import os

import numpy as np
import pytest
import torch

from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import PagedCache
from test_cache_abi import CHUNKS, FAKE, INV, UNS, _append, _cache


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_17074_amd import build
        build.build()
    return B.load()


def _rotation(**kw):
    r = B.SpecRotation()
    r.rotary_dim, r.num_q_heads = 128, 8
    r.freq = r.q = r.q_out = FAKE
    r.q_stride_tok = r.out_stride_tok = 1024
    r.q_stride_head = r.out_stride_head = 128
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _call(rotation=None, chunks=None, cache=None, args=None):
    return B.spec_cache_append_rotated(chunks or B.make_chunks(*CHUNKS), cache or _cache(), args or _append(),
                                       rotation or _rotation(), 0)


@pytest.mark.parametrize("kw,expect", [
    (dict(rotary_dim=0), INV), (dict(rotary_dim=-2), INV), (dict(rotary_dim=63), INV), (dict(rotary_dim=130), INV),
    (dict(interleaved=2), INV), (dict(freq=None), INV), (dict(freq=FAKE + 2), INV), (dict(positions=FAKE + 1), INV),
    (dict(rotary_dim=24), UNS), (dict(rotary_dim=8), UNS), (dict(rotary_dim=12, interleaved=1), UNS),
    (dict(num_q_heads=-1), INV), (dict(q=None), INV), (dict(q_out=None), INV), (dict(q=FAKE + 8), INV),
    (dict(q_out=FAKE + 2), INV), (dict(q_stride_tok=0), INV), (dict(q_stride_head=12), INV),
    (dict(out_stride_tok=1020), INV), (dict(out_stride_tok=512), INV), (dict(out_stride_head=64), INV),
    (dict(out_stride_tok=2048), INV),                                  # in place with strides of its own
    (dict(num_q_heads=1 << 20, out_stride_tok=1 << 28, q_stride_tok=1 << 28), UNS),
    (dict(q_stride_head=1 << 36, q=2 * FAKE), UNS),
])
def test_rotations_refused(kw, expect):
    assert _call(_rotation(**kw)) == expect


def test_heads_wider_than_the_angles_room_are_refused():
    wide = _cache(head_dim=1024, kv_stride_tok=2048, kv_stride_head=1024)
    args = _append(new_stride_tok=2048, new_stride_head=1024)
    assert _call(_rotation(rotary_dim=1024, num_q_heads=0), cache=wide, args=args) == UNS


def test_what_an_append_refuses():
    assert _call(args=_append(num_layers=2)) == INV                    # queries belong to one layer
    assert _call(args=_append(layer=2)) == INV
    assert _call(args=_append(k_new=None)) == INV
    assert _call(args=_append(new_stride_tok=4)) == INV
    assert _call(chunks=B.make_chunks([639], [2])) == INV
    assert _call(cache=_cache(block_table=None)) == INV
    assert B.spec_cache_append_rotated(B.make_chunks(*CHUNKS), _cache(), _append(), None, 0) == INV


def test_nothing_new_is_nothing_to_do():
    none = B.make_chunks([5, 7], [0, 0])
    assert _call(_rotation(q=None, q_out=None, freq=None), chunks=none) == B.SPEC_OK


def _paged():
    k = torch.zeros((2, 4, 32, 2, 64), dtype=torch.bfloat16)
    return PagedCache(k, k.clone(), torch.zeros((2, 2), dtype=torch.int32))


def test_arguments_of_the_method():
    c, chunks = _paged(), B.make_chunks([0, 5], [3, 2])
    new = torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    q = torch.zeros((5, 4, 64), dtype=torch.bfloat16)
    freq = torch.ones(32)
    bad = [
        dict(freq=freq.double()), dict(freq=freq[None]), dict(freq=torch.ones(64)[::2]),
        dict(q=q), dict(q_out=q), dict(q=q[:4], q_out=q), dict(q=q, q_out=q[:4]), dict(q=q.float(), q_out=q),
        dict(q=q, q_out=q[:, :2]), dict(q=q, q_out=torch.zeros((5, 4, 128), dtype=torch.bfloat16)[..., ::2]),
        dict(q=q[..., :32], q_out=q[..., :32]), dict(positions=torch.zeros(5)),
        dict(positions=torch.zeros(4, dtype=torch.int32)), dict(positions=torch.zeros(10, dtype=torch.int32)[::2]),
        dict(k_new=new[:4], v_new=new[:4]),
    ]
    for kw in bad:
        args = dict(k_new=new, v_new=new, freq=freq)
        args.update(kw)
        with pytest.raises(ValueError):
            c.append_rotated(chunks, **args)
    two = torch.zeros((2, 5, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="one layer"):
        c.append_rotated(chunks, two, two, freq, q, q)
    with pytest.raises(ValueError, match="device memory"):             # pools of the host
        c.append_rotated(chunks, new, new, freq, q, q)
    assert np.all(c.k.float().numpy() == 0)


@pytest.mark.parametrize("kw,expect", [
    # 70 tokens of 8 heads: heads behind each other are no overlap, so that what is refused is q's stride
    (dict(out_stride_tok=128, out_stride_head=70 * 128), UNS), (dict(out_stride_tok=160, out_stride_head=69 * 160 + 128), UNS),
    (dict(out_stride_tok=7 * 160 + 128, out_stride_head=160), UNS), (dict(out_stride_tok=1 << 33, out_stride_head=128), UNS),
    (dict(out_stride_tok=120, out_stride_head=70 * 128), INV), (dict(out_stride_tok=128, out_stride_head=69 * 128), INV),
    (dict(out_stride_tok=160, out_stride_head=69 * 160 + 120), INV), (dict(out_stride_tok=512, out_stride_head=128), INV),
    (dict(out_stride_tok=7 * 160 + 120, out_stride_head=160), INV), (dict(out_stride_tok=1000, out_stride_head=1000), INV),
])
def test_orders_of_the_rotated_queries(kw, expect):
    assert _call(_rotation(q=2 * FAKE, q_stride_head=1 << 36, **kw)) == expect
