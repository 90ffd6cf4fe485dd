"""The acceptance of drafted paths (stom_kv_accept) against the same rules kept in Python; everything is whole numbers or
moved bits, and has to be equal."""
import numpy as np
import pytest
import torch

import _kv as K
import _tree as T

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def _lib():
    from paper_2510_18269_b200 import oqm
    oqm.lib()
    return oqm


def _draft(rng, parents, vocab):
    return rng.integers(0, vocab, len(parents)), rng.integers(0, vocab, len(parents))


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _run(s, page, first, parent, draft, chosen, flag=0, rows=None):
    oqm = _lib()
    rows = len(draft) if rows is None else rows
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    path = torch.full((rows,), 7, dtype=torch.int32, device="cuda")
    count, following = (torch.full((len(first) - 1,), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"], s["refs"])
    oqm.stom_kv_accept(pool, seqs, _ints(first), _ints(draft), _ints(chosen), path, count, following,
                       parent=None if parent is None else _ints(parent), dev_flags=flags)
    torch.cuda.synchronize()
    assert flags.item() == flag
    return path.cpu().numpy(), count.cpu().numpy(), following.cpu().numpy()


def _same(s, book):
    assert np.array_equal(s["table"].cpu().numpy(), book.table)
    assert s["len"].tolist() == list(book.len)
    assert np.array_equal(s["refs"].cpu().numpy(), book.refs)
    assert torch.equal(s["k"], book.k) and torch.equal(s["v"], book.v)


def _book(s, lens, page):
    return K.Book(s["table_host"], lens, s["refs"].cpu().numpy(), page, s["k"], s["v"])


@pytest.mark.parametrize("had,new,page,layers,heads,d,dtype,kind,vocab", [
    ([0], [1], 16, 1, 2, 64, BF, "path", 2),                      # the only token there is
    ([700], [64], 50, 28, 4, 128, BF, "tree", 2),
    ([700], [64], 50, 3, 4, 128, BF, "path", 1),                  # all of a path: nothing moves
    ([10], [256], 16, 2, 2, 64, HF, "tree", 1),                   # the largest tree, every guess right
    ([10], [256], 1, 1, 1, 256, HF, "path", 1),
    ([31, 0, 15, 16, 17], [5, 9, 0, 30, 1], 16, 5, 2, 128, BF, "tree", 2),
    ([31, 0, 15, 16, 17], [5, 9, 0, 30, 1], 7, 2, 3, 64, HF, "forest", 2),
    ([100, 20], [40, 33], 1, 4, 2, 128, BF, "star", 30),          # pages of one token: many are given back
    ([3, 50, 0, 8] * 40, [3, 0, 12, 20] * 40, 8, 2, 2, 64, BF, "tree", 2),
    ([5], [100], 128, 60, 8, 256, BF, "tree", 1),
])
@pytest.mark.parametrize("order", ["token", "head"])
def test_paths(had, new, page, layers, heads, d, dtype, kind, vocab, order):
    rng = np.random.default_rng(len(had) * 7 + page)
    lens = [a + b for a, b in zip(had, new)]
    s = K.paged(rng, lens, page, layers, heads, d, dtype, order=order)
    first = np.concatenate([[0], np.cumsum(new)]).astype(int)
    parent = [p for n in new for p in T.a_tree(rng, n, kind)]
    draft, chosen = _draft(rng, parent, vocab)
    book = _book(s, lens, page)
    want = T.accept(book, first, parent, draft, chosen)
    got = _run(s, page, first, parent, draft, chosen)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)
    _same(s, book)


def test_a_draft_without_parents():
    rng = np.random.default_rng(5)
    for right in (0, 1, 4, 7):
        s = K.paged(rng, [37], 16, 2, 2, 64, BF)
        draft = np.arange(8)
        chosen = np.where(np.arange(8) < right, np.arange(8) + 1, 99)
        book = _book(s, [37], 16)
        want = T.accept(book, [0, 8], None, draft, chosen)
        got = _run(s, 16, [0, 8], None, draft, chosen)
        assert got[1][0] == right + 1 == want[1][0] and got[2][0] == (99 if right < 7 else 99)
        for a, b in zip(got, want):
            assert np.array_equal(a, b)
        _same(s, book)


def test_of_two_guesses_alike_the_lower_is_kept_and_nothing_follows_no_token():
    rng = np.random.default_rng(6)
    s = K.paged(rng, [30], 16, 1, 2, 64, BF)
    book = _book(s, [30], 16)
    parent, draft = [-1, 0, 0, 0, 2], [5, 8, 9, 9, -1]
    chosen = [9, 1, -1, 2, 3]                                     # node 2 is followed by nothing, whatever node 4 holds
    want = T.accept(book, [0, 5], parent, draft, chosen)
    got = _run(s, 16, [0, 5], parent, draft, chosen)
    assert got[0].tolist() == [0, 2, -1, -1, -1] and got[1].tolist() == [2] and got[2].tolist() == [-1]
    assert np.array_equal(want[0], got[0])
    _same(s, book)


def test_a_captured_step_of_reserve_and_accept():
    oqm = _lib()
    rng = np.random.default_rng(8)
    s = K.paged(rng, [20, 33], 16, 2, 2, 64, BF, spare=9, width=6)
    base = [20, 33]
    new = [12, 18]
    first = [0, 12, 30]
    parent = [p for n in new for p in T.a_tree(rng, n, "tree")]
    draft, chosen = _draft(rng, parent, 2)
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"], s["refs"])
    ws = torch.empty(oqm.stom_kv_pages_workspace_bytes(pool, seqs), dtype=torch.uint8, device="cuda")
    f, p, d, c = _ints(first), _ints(parent), _ints(draft), _ints(chosen)
    want = torch.zeros(2, dtype=torch.int32, device="cuda")
    path, count, following = _ints([0] * 30), _ints([0, 0]), _ints([0, 0])
    book = _book(s, base, 16)

    def step():
        want.copy_(s["len"] + _ints(new) if not torch.cuda.is_current_stream_capturing() else s["len"] + more)
        oqm.stom_kv_reserve(pool, seqs, want, ws)
        oqm.stom_kv_accept(pool, seqs, f, d, c, path, count, following, parent=p)

    more = _ints(new)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    assert book.reserve([x + n for x, n in zip(base, new)])
    T.accept(book, first, parent, draft, chosen)
    _same(s, book)
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert book.reserve([x + n for x, n in zip(book.len, new)])
        w = T.accept(book, first, parent, draft, chosen)
        assert np.array_equal(path.cpu().numpy(), w[0]) and count.tolist() == list(w[1]) and following.tolist() == list(w[2])
        _same(s, book)


@pytest.mark.parametrize("what", ["falls", "beyond", "more than tokens", "too many", "longer than its row"])
def test_sequences_that_do_not_fit_stay_as_they_are(what):
    rng = np.random.default_rng(9)
    s = K.paged(rng, [30, 300], 16, 2, 2, 64, BF, width=19)
    before = {n: s[n].clone() for n in ("k", "v", "table", "refs", "len")}
    first = {"falls": [6, 2, 2], "beyond": [0, 0, 400], "more than tokens": [0, 31, 31], "too many": [0, 0, 257],
             "longer than its row": [0, 0, 5]}[what]
    if what == "longer than its row":
        s["len"][1] = before["len"][1] = 305
    draft = np.ones(300, np.int64)
    got = _run(s, 16, first, None, draft, draft, flag=1)
    for n, x in before.items():
        assert torch.equal(s[n], x), n
    assert (got[0] == 7).all() and got[1].tolist() == [0, 0] and got[2].tolist() == [-1, -1]


def test_pages_that_are_none_are_skipped():
    rng = np.random.default_rng(10)
    s = K.paged(rng, [60], 16, 2, 2, 64, BF)
    page3 = int(s["table"][0, 3])
    s["table"][0, 3] = 10 ** 6
    k = s["k"].clone()
    parent = [-1] + [0] * 28 + [0]                                 # 30 nodes at 30 .. 59; node 29 lies in the page that is none
    draft, chosen = np.arange(30), np.full(30, 29)
    got = _run(s, 16, [0, 30], parent, draft, chosen, flag=1)
    assert got[1][0] == 2 and s["len"].item() == 32
    assert torch.equal(s["k"], k) and s["refs"][page3].item() == 1 and s["table"][0].tolist()[2:] == [-1, -1]


def test_results_that_are_not_wanted():
    oqm = _lib()
    rng = np.random.default_rng(11)
    s = K.paged(rng, [30], 16, 2, 2, 64, BF)
    book = _book(s, [30], 16)
    parent, draft, chosen = T.a_tree(rng, 12, "tree"), np.zeros(12, int), np.zeros(12, int)
    T.accept(book, [0, 12], parent, draft, chosen)
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"], s["refs"])
    oqm.stom_kv_accept(pool, seqs, _ints([0, 12]), _ints(draft), _ints(chosen), parent=_ints(parent))
    torch.cuda.synchronize()
    _same(s, book)
