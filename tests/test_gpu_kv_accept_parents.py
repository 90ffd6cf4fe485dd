"""Parents that are none (outside -1 .. j - 1) in the acceptance of drafted paths: they count as the context and are flagged, as
in the attention of the same tree."""
import numpy as np
import pytest

import _kv as K
import _tree as T
from test_gpu_kv_accept import BF, _book, _run, _same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("where,bad", [(w, b) for w in (0, 2, 5) for b in (w, w + 1, 6, -2, -(1 << 31), (1 << 31) - 1)])
def test_parents_that_are_none_count_as_the_context_and_are_flagged(where, bad):
    rng = np.random.default_rng(3)
    s = K.paged(rng, [40, 33], 16, 2, 2, 64, BF)
    parent = [-1, 0, 1, 2, 3, 4] + [-1, 0, 1]
    draft = np.zeros(9, int)
    told = list(parent)
    told[where] = bad
    parent[where] = -1
    book = _book(s, [40, 33], 16)
    want = T.accept(book, [0, 6, 9], parent, draft, draft)
    got = _run(s, 16, [0, 6, 9], told, draft, draft, flag=1)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)
    _same(s, book)


def test_parents_of_nobody_are_not_looked_at():
    """Behind the last sequence, and of one that is skipped."""
    rng = np.random.default_rng(4)
    s = K.paged(rng, [40], 16, 2, 2, 64, BF)
    book = _book(s, [40], 16)
    want = T.accept(book, [0, 4], [-1, 0, 1, 2], np.zeros(4, int), np.zeros(4, int))
    got = _run(s, 16, [0, 4], [-1, 0, 1, 2, 99, -7], np.zeros(6, int), np.zeros(6, int))
    assert np.array_equal(got[0][:4], want[0]) and (got[0][4:] == 7).all() and np.array_equal(got[1], want[1])
    _same(s, book)
