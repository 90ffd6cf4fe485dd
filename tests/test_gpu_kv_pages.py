"""Pages of a cache (stom_kv_reserve, _fork, _free, _compact) against the same rules applied one after the other in
Python.  Everything is whole numbers and copies: equality."""
import numpy as np
import pytest
import torch

import _kv as K

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def _lib():
    from paper_2510_18269_b200 import oqm
    oqm.lib()
    return oqm


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Both:
    """A cache on the device and its book in Python."""

    def __init__(self, lens, page=16, layers=2, heads=2, d=64, dtype=BF, spare=8, width=None, order="token", seed=0):
        self.oqm = _lib()
        s = K.paged(np.random.default_rng(seed), lens, page, layers, heads, d, dtype, spare=spare, width=width,
                    order=order, seed=seed)
        self.s = s
        # what a row holds behind its pages is not read
        s["table_host"][s["table_host"] < 0] = -1
        self.book = K.Book(s["table_host"], lens, s["refs"].cpu().numpy(), page, s["k"], s["v"])
        self.pool, self.seqs = self.oqm.KvPool(s["k"], s["v"]), self.oqm.KvSeqs(s["table"], s["len"], s["refs"])
        need = self.oqm.stom_kv_pages_workspace_bytes(self.pool, self.seqs)
        self.ws_all = torch.full((need + 256,), 170, dtype=torch.uint8, device="cuda")
        self.ws = self.ws_all[:need]
        self.flags = torch.zeros(1, dtype=torch.int32, device="cuda")

    def check(self, flags=0):
        torch.cuda.synchronize()
        b, s = self.book, self.s
        held = np.array([b.held(n) for n in b.len])
        cols = np.arange(b.table.shape[1])[None] < held[:, None]
        assert s["len"].tolist() == b.len
        assert np.array_equal(np.where(cols, s["table"].cpu().numpy(), -1), np.where(cols, b.table, -1))
        assert np.array_equal(s["refs"].cpu().numpy(), b.refs)
        assert torch.equal(s["k"], b.k) and torch.equal(s["v"], b.v)
        assert self.flags.item() == flags
        assert (self.ws_all[self.ws.numel():] == 170).all()

    def reserve(self, want):
        self.oqm.stom_kv_reserve(self.pool, self.seqs, _i32(want), self.ws, dev_flags=self.flags)
        return self.book.reserve(want)

    def fork(self, parent):
        self.oqm.stom_kv_fork(self.pool, self.seqs, _i32(parent), dev_flags=self.flags)
        self.book.fork(parent)

    def free(self, drop):
        self.oqm.stom_kv_free(self.pool, self.seqs, _i32(drop), dev_flags=self.flags)
        self.book.free(drop)

    def compact(self, apart=False):
        s = self.s
        t, r = (torch.full_like(s["table"], 77), torch.full_like(s["refs"], 77)) if apart else (s["table"], s["refs"])
        n = _i32([-5])
        was = s["table"].clone(), s["refs"].clone()
        self.oqm.stom_kv_compact(self.pool, self.seqs, t, r, n, self.ws, dev_flags=self.flags)
        live = self.book.compact()
        torch.cuda.synchronize()
        assert n.item() == live
        if apart:
            assert torch.equal(was[0], s["table"]) and torch.equal(was[1], s["refs"])
            s["table"].copy_(t)
            s["refs"].copy_(r)


@pytest.mark.parametrize("page,dtype,d,order", [(16, BF, 64, "token"), (50, HF, 128, "head"), (1, BF, 256, "token"), (7, BF, 64, "head")])
def test_reserve_fork_free_compact_in_a_row(page, dtype, d, order):
    b = Both([33, 0, 100, 0, 16, 0, 0, 1], page=page, d=d, dtype=dtype, spare=60, width=130 // page + 3, order=order, seed=page)
    b.reserve([40, 3, 0, 0, 17, 0, 0, 1])                         # grows, begins, stays
    b.check()
    b.fork([-1, -1, -1, 2, -1, 0, 0, -1])                         # three candidates, two of them of the same parent
    b.check()
    b.reserve([41, 0, 0, 101, 0, 42, 41, 9])                      # all three holders of a page grow; only one child of 2 does
    b.check()
    b.free([0, 1, 0, 0, 1, 0, 1, 0])
    b.check()
    b.compact()
    b.check()
    b.reserve([60, 5, 101, 0, 1, 0, 7, 0])
    b.check()


def test_last_holder_keeps_the_page_and_one_that_stays_forces_a_copy():
    b = Both([10, 0, 0, 10, 0], spare=9)
    b.fork([-1, 0, 0, -1, 3])
    b.check()
    shared = int(b.s["table"][0, 0])
    b.reserve([11, 11, 11, 0, 11])
    b.check()
    t = b.s["table"].cpu().numpy()
    assert t[2, 0] == shared and t[0, 0] != shared and t[1, 0] != shared   # the last of the three keeps it
    assert t[4, 0] != t[3, 0]                                             # row 3 stays behind: row 4 copies


def test_full_last_page_is_shared_without_a_copy():
    b = Both([32, 0], spare=4, width=4)
    b.fork([-1, 0])
    b.reserve([33, 40])
    b.check()
    assert b.s["refs"].cpu().numpy()[b.book.table[0, :2]].tolist() == [2, 2]


def test_too_few_pages_change_nothing():
    oqm = _lib()
    b = Both([20, 0, 5], spare=3, width=10)
    assert not b.reserve([36, 16, 64])                            # 1 + 1 + 3 of 3
    b.check(flags=oqm.FLAG_NO_PAGE)
    b.flags.zero_()
    assert not b.reserve([160, 160, 160])                         # more than the pool has at all
    b.check(flags=oqm.FLAG_NO_PAGE)
    b.flags.zero_()
    assert b.reserve([33, 16, 17])                                # exactly three
    b.check()


def test_wishes_beyond_a_row_are_skipped():
    oqm = _lib()
    b = Both([20, 3], spare=9, width=3)
    b.reserve([49, 48])
    b.check(flags=oqm.FLAG_BAD_INDEX)
    b.flags.zero_()
    b.reserve([-7, 2 ** 31 - 1])
    b.check(flags=oqm.FLAG_BAD_INDEX)


def test_forks_that_cannot_be_are_skipped():
    oqm = _lib()
    b = Both([20, 0, 0, 0, 6], spare=9)
    before = b.s["table"].clone()
    # out of range twice, a parent that is forked itself, a row that is not empty; row 3 is fine
    for parent, fine in (([-1, 9, -1, -1, -1], False), ([-1, -3, -1, -1, -1], False), ([-1, 0, 1, -1, -1], True),
                         ([-1, -1, -1, -1, 0], False)):
        b.oqm.stom_kv_fork(b.pool, b.seqs, _i32(parent), dev_flags=b.flags)
        b.book.fork([p if -1 <= p < 5 and not (p >= 0 and parent[p] != -1) else -1 for p in parent])
        b.check(flags=oqm.FLAG_BAD_INDEX)
        b.flags.zero_()
        assert torch.equal(before, b.s["table"]) != fine
        before = b.s["table"].clone()
    b.fork([-1, -1, 4, 0, -1])
    b.check()


def test_bad_page_ids_are_skipped():
    oqm = _lib()
    b = Both([40, 0], spare=9)
    b.s["table"][0, 1], b.s["table"][0, 2] = -4, 10 ** 8
    refs = b.s["refs"].clone()
    b.oqm.stom_kv_reserve(b.pool, b.seqs, _i32([41, 0]), b.ws, dev_flags=b.flags)     # the partly filled page is none
    assert b.flags.item() == oqm.FLAG_BAD_INDEX and torch.equal(refs, b.s["refs"]) and b.s["len"].tolist() == [41, 0]
    b.flags.zero_()
    b.oqm.stom_kv_fork(b.pool, b.seqs, _i32([-1, 0]), dev_flags=b.flags)
    assert b.flags.item() == oqm.FLAG_BAD_INDEX and int(b.s["refs"].sum()) == int(refs.sum()) + 1
    b.flags.zero_()
    t = b.s["table"].clone()
    b.oqm.stom_kv_compact(b.pool, b.seqs, t, b.s["refs"].clone(), None, b.ws, dev_flags=b.flags)
    assert b.flags.item() == oqm.FLAG_BAD_INDEX and t[0, 1] == -4 and t[0, 2] == 10 ** 8
    b.flags.zero_()
    b.oqm.stom_kv_free(b.pool, b.seqs, _i32([1, 1]), dev_flags=b.flags)
    assert b.flags.item() == oqm.FLAG_BAD_INDEX and b.s["len"].tolist() == [0, 0] and (b.s["table"] == -1).all()
    assert int(b.s["refs"].sum()) == int(refs.sum()) - 1
    b.flags.zero_()
    # a table that says more than its counts: no count goes below zero
    b.s["table"][0, 0], b.s["len"][0] = int((b.s["refs"] == 0).nonzero()[0]), 5
    refs = b.s["refs"].clone()
    b.oqm.stom_kv_free(b.pool, b.seqs, _i32([1, 0]), dev_flags=b.flags)
    assert b.flags.item() == oqm.FLAG_BAD_INDEX and torch.equal(refs, b.s["refs"])


@pytest.mark.parametrize("apart", [False, True])
def test_compact(apart):
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 200, 30).tolist()
    b = Both(lens, page=7, layers=3, heads=1, d=64, spare=11, seed=2)
    b.free((rng.random(30) < 0.5).astype(int).tolist())
    b.fork([-1 if n else (i + 1) % 30 if b.book.len[(i + 1) % 30] else -1 for i, n in enumerate(b.book.len)])
    b.check()
    b.compact(apart)
    b.check()
    b.compact(apart)                                              # nothing left to move
    b.check()


def test_compact_of_an_empty_and_of_a_full_pool():
    b = Both([0, 0], spare=5)
    b.compact(True)
    b.check()
    b = Both([64, 64], spare=0)
    b.compact()
    b.check()


def test_many_rows_and_pages():
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 40, 3000).tolist()
    b = Both(lens, page=2, layers=1, heads=1, d=64, spare=20000, width=40, seed=4)
    full = [i for i, n in enumerate(lens) if n]
    b.fork([-1 if n else int(rng.choice(full)) for n in lens])
    b.check()
    done = b.reserve([n + int(rng.integers(0, 30)) for n in b.book.len])
    b.check(flags=0 if done else _lib().FLAG_NO_PAGE)
    b.flags.zero_()
    assert b.reserve([n + int(rng.integers(0, 12)) for n in b.book.len])
    b.check()
    b.free((rng.random(3000) < 0.3).astype(int).tolist())
    b.check()
    b.compact()
    b.check()


def test_most_rows_share_one_page():
    oqm = _lib()
    n = oqm_rows = 8192
    b = Both([5] + [0] * (n - 1), page=16, layers=1, heads=1, d=64, spare=n + 10, width=2)
    b.fork([-1] + [0] * (n - 1))
    b.reserve([6] * oqm_rows)
    b.check()


def test_captured_branching():
    """free, fork and reserve as one graph, replayed: a new set of candidates every time."""
    b = Both([20, 9, 0, 0, 0, 0], spare=16, width=4)
    drop, parent, want = _i32([0, 0, 1, 1, 1, 1]), _i32([-1, -1, 0, 0, 1, 1]), _i32([0, 0, 21, 21, 10, 10])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        b.oqm.stom_kv_free(b.pool, b.seqs, drop, dev_flags=b.flags)
        b.oqm.stom_kv_fork(b.pool, b.seqs, parent, dev_flags=b.flags)
        b.oqm.stom_kv_reserve(b.pool, b.seqs, want, b.ws, dev_flags=b.flags)
    for _ in range(3):
        g.replay()
        b.book.free(drop.tolist())
        b.book.fork(parent.tolist())
        b.book.reserve(want.tolist())
        b.check()
