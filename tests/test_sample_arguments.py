"""What sampling refuses, on a host without a GPU."""
import os

import pytest
import torch

from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.sample import Sampler

FAKE = 1 << 20      # a fake device address; never dereferenced on these paths
INV, UNS, WSP = B.SPEC_ERR_INVALID_ARG, B.SPEC_ERR_UNSUPPORTED, B.SPEC_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_17074_amd import build
        build.build()
    return B.load()


def _args(**kw):
    a = B.SpecSampleArgs()
    a.num_rows, a.vocab, a.dtype = 3, 1000, B.SPEC_F32
    a.logits = a.uniforms = a.tokens = FAKE
    a.logits_stride = a.rows_stride = 1000
    for k, v in kw.items():
        setattr(a, k, v)
    return a


PROBS = dict(rows_kind=B.SPEC_SAMPLE_PROBS, rows=2 * FAKE)


@pytest.mark.parametrize("kw,expect", [
    (dict(num_rows=0), INV), (dict(num_rows=-1), INV), (dict(vocab=0), INV), (dict(dtype=2), INV), (dict(rows_kind=3), INV),
    (dict(rows_kind=-1), INV), (dict(logits=None), INV), (dict(logits=FAKE + 2), INV), (dict(logits_stride=999), INV),
    (dict(temperature=FAKE + 2), INV), (dict(top_k=FAKE + 1), INV), (dict(top_p=FAKE + 2), INV), (dict(min_p=FAKE + 3), INV),
    (dict(uniforms=None), INV), (dict(uniforms=FAKE + 2), INV), (dict(tokens=FAKE + 2), INV),
    (dict(tokens=None), INV),                                                # nothing to do
    (dict(PROBS, rows=None), INV), (dict(PROBS, rows=FAKE + 2), INV), (dict(PROBS, rows_stride=999), INV),
    (dict(PROBS, rows=FAKE, rows_stride=1004), INV),                         # in place with another stride
    (dict(vocab=(1 << 28) + 1, logits_stride=1 << 30), UNS), (dict(num_rows=1 << 22), UNS),
])
def test_refused(kw, expect):
    assert B.spec_sample(_args(**kw), FAKE, 1 << 30, 0) == expect
    assert B.spec_sample_workspace_bytes(_args(**kw))[0] == expect


@pytest.mark.parametrize("kw", [
    dict(), dict(num_rows=1, logits_stride=0), PROBS, dict(PROBS, tokens=None, uniforms=None), dict(PROBS, rows=FAKE),
    dict(dtype=B.SPEC_BF16, logits=FAKE + 2), dict(num_rows=(1 << 22) - 1),
])
def test_accepted(kw):
    assert B.spec_sample_workspace_bytes(_args(**kw))[0] == B.SPEC_OK


@pytest.mark.parametrize("ws,size", [(None, 1 << 30), (FAKE + 16, 1 << 30), (FAKE, 100)])
def test_workspaces_refused(ws, size):
    assert B.spec_sample(_args(), ws, size, 0) == WSP


def test_workspaces_of_long_rows():
    """A row's runs of ids, lists and histograms: bounded whatever its length."""
    for rows, vocab in ((1, 1), (1, 1 << 28), (1000, 50), (3, 128256), (256, 128256), (257, 1 << 20)):
        st, need = B.spec_sample_workspace_bytes(_args(num_rows=rows, vocab=vocab, logits_stride=1 << 30))
        assert st == B.SPEC_OK and 0 < need <= rows * (512 + 8192 + 8 * 33280) + 256


def test_null_arguments():
    import ctypes as C
    assert B.load().spec_sample(None, None, 0, None) == INV
    assert B.load().spec_sample_workspace_bytes(C.byref(_args()), None) == INV


def test_arguments_of_the_method():
    s = Sampler("cpu")
    x, u, t = torch.zeros((3, 10)), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    bad = [
        dict(logits=x[0]), dict(logits=x.double()), dict(logits=x[:0]), dict(logits=torch.zeros((3, 20))[:, ::2]),
        dict(uniforms=None), dict(uniforms=u.double()), dict(uniforms=u[:2]), dict(uniforms=torch.zeros(6)[::2]),
        dict(tokens=t.long()), dict(tokens=t[:2]), dict(temperature=t), dict(temperature=torch.zeros(4)), dict(top_k=u),
        dict(top_k=t.long()), dict(top_p=u.half()), dict(min_p=u[None]), dict(probs=x[:2]), dict(probs=x.bfloat16()),
        dict(probs=torch.zeros((3, 20))[:, ::2]), dict(probs=x, kept_logits=x.clone()),
    ]
    for kw in bad:
        args = dict(logits=x, uniforms=u, tokens=t)
        args.update(kw)
        with pytest.raises(ValueError):
            s.run(**args)
    with pytest.raises(ValueError, match="device memory"):
        s.run(x, u, t)
