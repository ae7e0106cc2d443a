"""The page bookkeeping (host code) against a plain model of it."""
import ctypes as C

import numpy as np
import pytest

from paper_2505_17074_amd import binding as B
from paper_2505_17074_amd.cache import Pages


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_17074_amd import build
        build.build()
    return B.load()


class Model:
    """Lists and counts, with the rules written out."""

    def __init__(self, n, P):
        self.n, self.P, self.holders, self.seqs = n, P, [0] * n, {}

    def free(self):
        return [x for x in range(self.n) if self.holders[x] == 0]

    def open(self):
        s = next(i for i in range(len(self.seqs) + 1) if i not in self.seqs)
        self.seqs[s] = [0, []]
        return s

    def resize(self, s, tokens):
        old, pages = self.seqs[s]
        want = -(-tokens // self.P)
        copy = None
        if tokens > old:
            apart = old % self.P != 0 and self.holders[pages[-1]] > 1
            if want - len(pages) + apart > len(self.free()):
                return "full"
            if apart:
                new = self.free()[0]
                copy = (pages[-1], new, old % self.P)
                self.holders[pages[-1]] -= 1
                self.holders[new] = 1
                pages[-1] = new
            while len(pages) < want:
                new = self.free()[0]
                self.holders[new] = 1
                pages.append(new)
        else:
            while len(pages) > want:
                self.holders[pages.pop()] -= 1
        self.seqs[s][0] = tokens
        return copy

    def fork(self, s):
        c = self.open()
        self.seqs[c] = [self.seqs[s][0], list(self.seqs[s][1])]
        for x in self.seqs[s][1]:
            self.holders[x] += 1
        return c

    def close(self, s):
        for x in self.seqs.pop(s)[1]:
            self.holders[x] -= 1

    def compact(self):
        used = self.n - len(self.free())
        to = [x for x in range(used) if self.holders[x] == 0]
        src = [x for x in range(self.n - 1, used - 1, -1) if self.holders[x] > 0]
        out = []
        for a, b in zip(src, to):
            rows = max(min(self.P, t - j * self.P) for t, pg in self.seqs.values() for j, x in enumerate(pg) if x == a)
            out.append([a, b, rows])
            self.holders[b], self.holders[a] = self.holders[a], 0
            for q in self.seqs.values():
                q[1][:] = [b if x == a else x for x in q[1]]
        return out


@pytest.mark.parametrize("seed", range(6))
def test_against_the_model(seed):
    rng = np.random.default_rng(seed)
    n, P = int(rng.choice([1, 5, 40, 64, 65, 200])), int(rng.choice([32, 64, 96]))
    a, b = Pages(n, P), Model(n, P)
    for _ in range(600):
        what = rng.choice(["open", "resize", "resize", "resize", "fork", "close", "compact"])
        live = sorted(b.seqs)
        if what == "open" and len(live) < 12 or not live:
            assert a.open() == b.open()
        elif what == "resize":
            s = int(rng.choice(live))
            t = int(rng.integers(0, max(2, n * P // 2)))
            want = b.resize(s, t)
            if want == "full":
                with pytest.raises(B.SpecError) as e:
                    a.resize(s, t)
                assert e.value.status == B.SPEC_ERR_NO_PAGES
            else:
                assert a.resize(s, t) == want
        elif what == "fork" and len(live) < 12:
            s = int(rng.choice(live))
            assert a.fork(s) == b.fork(s)
        elif what == "close":
            s = int(rng.choice(live))
            a.close(s)
            b.close(s)
        elif what == "compact":
            assert a.compact().tolist() == b.compact()
        assert a.free == len(b.free())
        for s, (_, pages) in b.seqs.items():
            assert a.table(s).tolist() == pages


def test_a_fork_copies_only_what_it_will_overwrite():
    p = Pages(10, 32)
    a = p.open()
    assert p.resize(a, 40) is None and p.table(a).tolist() == [0, 1]
    b = p.fork(a)
    assert p.resize(b, 41) == (1, 2, 8) and p.table(b).tolist() == [0, 2]
    assert p.resize(a, 41) is None                       # page 1 is its own again
    c = p.fork(a)
    p.resize(c, 32)
    assert p.resize(c, 33) is None and p.table(c).tolist() == [0, 3]   # behind a full page: no copy
    p.close(a)
    p.close(b)
    assert p.free == 8 and p.table(c).tolist() == [0, 3]
    assert p.compact().tolist() == [[3, 1, 1]] and p.table(c).tolist() == [0, 1]


def test_refusals():
    L = B.load()
    h, i32, cp = C.c_void_p(), C.c_int32(), B.SpecPageCopy()
    for n, P in ((0, 64), (-1, 64), (4, 0), (4, 16), (4, 48), (4, -32)):
        assert L.spec_pages_create(n, P, C.byref(h)) == B.SPEC_ERR_INVALID_ARG
    assert L.spec_pages_create(4, 64, None) == B.SPEC_ERR_INVALID_ARG
    assert L.spec_pages_create(4, 64, C.byref(h)) == B.SPEC_OK
    assert L.spec_pages_open(h, None) == B.SPEC_ERR_INVALID_ARG
    assert L.spec_pages_open(h, C.byref(i32)) == B.SPEC_OK and i32.value == 0
    for s in (-1, 1, 1 << 30):
        assert L.spec_pages_resize(h, s, 5, C.byref(cp)) == B.SPEC_ERR_INVALID_ARG
        assert L.spec_pages_fork(h, s, C.byref(i32)) == B.SPEC_ERR_INVALID_ARG
        assert L.spec_pages_close(h, s) == B.SPEC_ERR_INVALID_ARG
        assert L.spec_pages_table(h, s, None, 0, C.byref(i32)) == B.SPEC_ERR_INVALID_ARG
    assert L.spec_pages_resize(h, 0, -1, C.byref(cp)) == B.SPEC_ERR_INVALID_ARG
    assert L.spec_pages_resize(h, 0, 5, None) == B.SPEC_ERR_INVALID_ARG
    assert L.spec_pages_resize(h, 0, 257, C.byref(cp)) == B.SPEC_ERR_NO_PAGES
    assert L.spec_pages_resize(h, 0, 2**31 - 1, C.byref(cp)) == B.SPEC_ERR_NO_PAGES
    assert L.spec_pages_free_count(h) == 4
    assert L.spec_pages_resize(h, 0, 256, C.byref(cp)) == B.SPEC_OK
    out = (C.c_int32 * 4)()
    assert L.spec_pages_table(h, 0, out, 3, C.byref(i32)) == B.SPEC_ERR_WORKSPACE and i32.value == 4
    assert L.spec_pages_table(h, 0, out, 4, C.byref(i32)) == B.SPEC_OK and list(out) == [0, 1, 2, 3]
    # a fork of a partly filled page that has no page left for its copy: nothing changes
    assert L.spec_pages_resize(h, 0, 250, C.byref(cp)) == B.SPEC_OK
    assert L.spec_pages_fork(h, 0, C.byref(i32)) == B.SPEC_OK and i32.value == 1
    assert L.spec_pages_resize(h, 1, 251, C.byref(cp)) == B.SPEC_ERR_NO_PAGES
    assert L.spec_pages_table(h, 1, out, 4, C.byref(i32)) == B.SPEC_OK and list(out) == [0, 1, 2, 3]
    assert L.spec_pages_resize(h, 0, 100, C.byref(cp)) == B.SPEC_OK
    assert L.spec_pages_close(h, 1) == B.SPEC_OK and L.spec_pages_free_count(h) == 2
    b = B.SpecPageCopy()
    assert L.spec_pages_compact(h, C.byref(b), 0, C.byref(i32)) == B.SPEC_OK and i32.value == 0
    assert L.spec_pages_compact(h, None, -1, C.byref(i32)) == B.SPEC_ERR_INVALID_ARG
    for f in (L.spec_pages_open, L.spec_pages_close):
        assert f(None, None if f is L.spec_pages_open else 0) == B.SPEC_ERR_INVALID_ARG
    assert L.spec_pages_free_count(None) == 0
    L.spec_pages_destroy(h)
    L.spec_pages_destroy(None)


def test_compact_says_how_much_room_it_needs():
    p = Pages(6, 32)
    a, b = p.open(), p.open()
    p.resize(a, 64)
    p.resize(b, 64)
    p.close(a)
    n, out = C.c_int32(), B.SpecPageCopy()
    assert p._lib.spec_pages_compact(p._h, C.byref(out), 1, C.byref(n)) == B.SPEC_ERR_WORKSPACE and n.value == 2
    assert p.table(b).tolist() == [2, 3]
    assert p.compact().tolist() == [[3, 0, 32], [2, 1, 32]] and p.table(b).tolist() == [1, 0]
