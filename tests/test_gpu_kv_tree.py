"""Attention of several new tokens per sequence over a paged cache (stom_kv_attend_tree) against softmax attention in 64 bits.

Tolerance of out, element by element, with u the type's half step (2^-8 bf16, 2^-11 fp16):
    u |out|                         the one rounding of the result
  + mean_w|V| * (u + u^2 + 2^-15)   the weights' rounding to the type (u of each), its product with the result's, and scores,
                                    exponentials and sums in binary32 as for one new token: scores below 32 in magnitude
                                    carry below 2^-16 from their sum and scaling, the exponential doubles it at most
  + 2^-24 (fp16)                    where the result is subnormal
lse: 2^-15 absolute by the same sum, plus 2^-22 relative."""
import math

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


def _close(got, want, mag, dtype):
    u = K.HALF_STEP[dtype]
    lim = u * np.abs(want) + mag * (u + u * u + 2.0 ** -15) + (2.0 ** -24 if dtype is HF else 0.0)
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    bad = np.abs(got - want) > lim
    assert not bad.any(), (int(bad.sum()), float(np.max(np.abs(got - want) / np.maximum(lim, 1e-30))))


def _close_lse(got, want):
    got = got.double().cpu().numpy()
    empty = want == -np.inf
    assert (got[empty] == -np.inf).all()
    assert (np.abs(got - np.where(empty, 0.0, want))[~empty] <= 2.0 ** -15 + 2.0 ** -22 * np.abs(want[~empty])).all()


def _make(had, new, hq, hk, d, page, dtype, kind="tree", order="token", layers=1, seed=0, extra=0, width=None):
    rng = np.random.default_rng(seed)
    lens = [a + b for a, b in zip(had, new)]
    s = K.paged(rng, lens, page, layers, hk, d, dtype, order=order, seed=seed, width=width)
    first = [int(x) for x in np.concatenate([[0], np.cumsum(new)])]
    parent = None if kind == "chain" else [p for n in new for p in T.a_tree(rng, n, kind)]
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    rows = first[-1] + extra
    s.update(lens=lens, first=first, parent=parent, rows=rows, q=(1.5 * torch.randn(rows, hq, d, generator=g, device="cuda")).to(dtype))
    return s


def _call(s, scale=None, cap=0.0, window=0, layer=0, with_lse=True, q=None, out=None, flag=0, stream=None):
    oqm = _lib()
    q = s["q"] if q is None else q
    out = torch.full_like(s["q"], 7.0) if out is None else out
    rows, hq, d = q.shape
    lse = torch.full((rows, hq), 7.0, device="cuda") if with_lse else None
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"])
    ints = lambda x: None if x is None else torch.tensor(list(x) + [-1] * (rows - len(x)), dtype=torch.int32, device="cuda")  # noqa: E731
    need = oqm.stom_kv_attend_tree_workspace_bytes(pool, seqs, rows, hq)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    first = torch.tensor(s["first"], dtype=torch.int32, device="cuda")
    oqm.stom_kv_attend_tree(pool, seqs, layer, first, q, out, scale or d ** -0.5, ws[:need], parent=ints(s["parent"]), lse=lse,
                            softcap=cap, window=window, dev_flags=flags, stream=stream)
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all() and flags.item() == flag
    return out, lse


def _check(s, out, lse, scale=None, cap=0.0, window=0, layer=0, q=None, dtype=None):
    q = s["q"] if q is None else q
    n = s["first"][-1]
    want, wlse, mag = T.attend_nodes(s["k"], s["v"], s["table_host"], s["lens"], s["first"], s["parent"], q, scale or q.shape[2] ** -0.5,
                                     cap, window, layer)
    assert np.abs(wlse[:n][np.isfinite(wlse[:n])]).max(initial=0.0) < 32
    _close(out[:n], want[:n], mag[:n], q.dtype)
    assert (out[n:] == 7.0).all()                                  # rows of no sequence
    if lse is not None:
        _close_lse(lse[:n], wlse[:n])
        assert (lse[n:] == 7.0).all()


SHAPES = [
    ([0], [1], 4, 4, 64, 16, BF, "path"),                          # the first token there is
    ([100], [1], 4, 2, 128, 16, BF, "path"),                       # one token, as a decode step
    ([0], [9], 8, 2, 64, 4, HF, "tree"),                           # a tree without a context
    ([127, 128, 129, 0, 1], [1, 2, 3, 4, 5], 8, 2, 64, 16, HF, "tree"),   # around a tile's end
    ([12583], [5], 28, 4, 128, 50, BF, "path"),                    # one stream over the whole device
    ([2500], [64], 28, 4, 128, 50, BF, "tree"),                    # more rows than a tile
    ([700, 3, 0, 1201, 50], [7, 0, 12, 33, 1], 28, 4, 128, 50, BF, "forest"),   # a sequence without new tokens between
    ([333, 64, 129], [20, 19, 18], 16, 2, 128, 1, HF, "tree"),     # pages of one token
    ([333, 64, 1000], [11, 3, 30], 12, 1, 128, 7, BF, "star"),     # 12 query heads on one kv head, odd pages
    ([90, 400], [17, 5], 12, 1, 64, 33, HF, "roots"),
    ([513, 30], [6, 9], 64, 1, 64, 64, BF, "tree"),                # the largest group
    ([300, 77, 5, 0], [40, 1, 9, 3], 8, 4, 256, 16, BF, "tree"),
    ([513, 30], [13, 20], 20, 1, 256, 64, HF, "forest"),
    ([200], [256], 4, 2, 128, 50, BF, "tree"),                     # the largest tree
    ([61], [255], 2, 2, 64, 16, HF, "path"),
    ([5, 9, 2, 0, 31] * 40, [1, 0, 3, 2, 5] * 40, 4, 2, 64, 4, BF, "tree"),     # 200 short ones
]


@pytest.mark.parametrize("had,new,hq,hk,d,page,dtype,kind", SHAPES)
def test_trees(had, new, hq, hk, d, page, dtype, kind):
    s = _make(had, new, hq, hk, d, page, dtype, kind)
    _check(s, *_call(s))


@pytest.mark.parametrize("had,new,hq,hk,d,page,dtype", [
    ([0], [1], 4, 2, 64, 16, BF), ([0], [300], 8, 2, 128, 16, HF), ([1000, 0, 77], [129, 600, 1], 14, 2, 128, 50, BF),
    ([64], [511], 3, 3, 256, 64, BF), ([3000], [333], 7, 1, 64, 128, HF),
])
def test_chains(had, new, hq, hk, d, page, dtype):
    s = _make(had, new, hq, hk, d, page, dtype, "chain")
    _check(s, *_call(s))


@pytest.mark.parametrize("kind", ["tree", "path", "chain", "roots"])
@pytest.mark.parametrize("window,cap,d,dtype", [(1, 0.0, 64, BF), (3, 5.0, 128, HF), (100, 0.0, 128, BF), (128, 30.0, 256, BF),
                                                (5000, 0.0, 64, HF)])
def test_windows_and_caps(kind, window, cap, d, dtype):
    s = _make([250, 0, 130, 3], [20, 9, 1, 40], 8, 2, d, 16, dtype, kind, seed=window)
    _check(s, *_call(s, cap=cap, window=window), cap=cap, window=window)


@pytest.mark.parametrize("cap", [0.0, 4.0, 30.0])
@pytest.mark.parametrize("scale,d,dtype", [(-0.09, 128, BF), (0.2, 64, HF), (1e-20, 256, HF), (-0.06, 256, BF)])
def test_scales_of_either_sign(scale, cap, d, dtype):
    s = _make([250, 0, 130, 3], [20, 9, 1, 40], 8, 2, d, 16, dtype, "tree", seed=d)
    for window in (0, 40):
        _check(s, *_call(s, scale=scale, cap=cap, window=window), scale=scale, cap=cap, window=window)


def test_a_chain_without_parents_equals_one_with():
    s = _make([777, 5], [30, 100], 8, 2, 128, 16, BF, "path")
    a = _call(s)
    s["parent"] = None
    b = _call(s)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_the_same_call_gives_the_same_bits():
    s = _make([2000, 30, 511], [40, 7, 90], 28, 4, 128, 50, BF)
    a, b = _call(s), _call(s)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("d,hq,hk,page,dtype", [(128, 64, 8, 16, HF), (64, 16, 2, 50, BF), (256, 8, 4, 64, BF)])
def test_many_units_a_block_again_and_again(d, hq, hk, page, dtype):
    """Blocks go through many short units, warps at their own pace: every call gives the bits of the first, which are right."""
    rng = np.random.default_rng(d)
    had, new = rng.integers(0, 2000, 40).tolist(), rng.integers(1, 34, 40).tolist()
    s = _make(had, new, hq, hk, d, page, dtype)
    out, lse = _call(s)
    for _ in range(15):
        again = _call(s)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    keep = {0: s["first"][0], 20: s["first"][20], 39: s["first"][39]}
    want, wlse, mag = T.attend_nodes(s["k"], s["v"], s["table_host"][list(keep)], [s["lens"][i] for i in keep],
                                     [0] + np.cumsum([new[i] for i in keep]).tolist(),
                                     [p for i in keep for p in s["parent"][s["first"][i]:s["first"][i + 1]]],
                                     torch.cat([s["q"][s["first"][i]:s["first"][i + 1]] for i in keep]), d ** -0.5)
    rows = [r for i in keep for r in range(s["first"][i], s["first"][i + 1])]
    _close(out[rows], want, mag, dtype)
    _close_lse(lse[rows], wlse)


@pytest.mark.parametrize("order", ["token", "head"])
def test_layers_strides_and_rows_behind_the_last_sequence(order):
    s = _make([150, 64], [10, 3], 8, 4, 128, 16, BF, order=order, layers=3, extra=5)
    wide = torch.full((18, 8, 2 * 128), 7.0, dtype=BF, device="cuda")
    q = torch.zeros(18, 9, 128, dtype=BF, device="cuda")[:, 1:]
    q.copy_(s["q"])
    out, lse = _call(s, layer=2, q=q, out=wide[..., 128:])
    _check(s, out, lse, layer=2, q=q)
    assert (wide[..., :128] == 7.0).all()
    out2, none = _call(s, layer=2, with_lse=False)
    assert none is None and torch.equal(out2, out)


def test_no_token_no_sequence():
    s = _make([30, 40], [0, 0], 4, 2, 64, 16, BF, extra=2)
    out, lse = _call(s)
    assert (out == 7.0).all() and (lse == 7.0).all()
    s = _make([30], [2], 4, 2, 64, 16, BF)
    s["q"] = s["q"][:0]
    s["first"], s["parent"] = [0, 0], []
    _call(s)


def test_first_may_begin_behind_row_0():
    s = _make([30, 40], [3, 4], 4, 2, 64, 16, BF, extra=6)
    out, lse = _call(s)
    t = dict(s, first=[x + 2 for x in s["first"]], parent=[9, 9] + s["parent"], q=torch.cat([s["q"][-2:], s["q"][:-2]]))
    out2, lse2 = _call(t)
    assert torch.equal(out2[2:9], out[:7]) and torch.equal(lse2[2:9], lse[:7])
    assert (out2[:2] == 7.0).all() and (out2[9:] == 7.0).all()


@pytest.mark.parametrize("what", ["falls", "beyond", "negative", "more than tokens", "too many"])
def test_sequences_that_do_not_fit_are_skipped_and_flagged(what):
    kind = "tree"
    s = _make([50, 300, 60], [4, 6, 5], 4, 2, 64, 16, BF, kind, extra=300)
    good = _call(s)
    t = dict(s)
    if what == "falls":
        t["first"] = [0, 10, 4, 15]                                # sequence 0: 10 rows (it has 54 tokens), 1: none, 2: 11
        t["parent"] = s["parent"][:4] + [-1] * 11
        rows = slice(0, 4)                                         # of these, only sequence 1 is out of order
        out, lse = _call(t, flag=1)
        assert (out[15:] == 7.0).all()
        return
    if what == "beyond":
        t["first"] = [0, 4, 10, 400]
        out, lse = _call(t, flag=1)
        rows = slice(0, 10)
    elif what == "negative":
        t["first"] = [-4, 4, 10, 15]
        out, lse = _call(t, flag=1)
        rows = slice(4, 15)
    elif what == "more than tokens":
        t["len"] = s["len"].clone()
        t["len"][0] = 3
        out, lse = _call(t, flag=1)
        rows = slice(4, 15)
    else:
        t["first"] = [0, 4, 10, 10 + 257]                          # 257 nodes, and a length that has them
        t["len"] = s["len"].clone()
        t["len"][2] = 300
        t["table"] = s["table"].clone()
        out, lse = _call(t, flag=1)
        rows = slice(0, 10)
    assert torch.equal(out[rows], good[0][rows]) and torch.equal(lse[rows], good[1][rows])
    rest = torch.ones(out.shape[0], dtype=torch.bool)
    rest[rows] = False
    assert (out[rest.cuda()] == 7.0).all()


def test_parents_that_are_none_count_as_the_context():
    s = _make([40], [6], 4, 2, 64, 16, BF)
    for bad in (2, 5, -2, 1 << 30):
        t = dict(s, parent=[-1, 0, bad, 1, 2, 0])
        out, lse = _call(t, flag=1)
        _check(dict(s, parent=[-1, 0, -1, 1, 2, 0]), out, lse)


def test_pages_that_are_none_are_absent_and_flagged():
    s = _make([100, 60], [5, 30], 4, 2, 128, 16, BF)
    for where, value in (((0, 2), -1), ((0, 6), 10 ** 6), ((1, 0), -7), ((1, 4), 10 ** 9)):
        t = dict(s, table=s["table"].clone(), table_host=s["table_host"].copy())
        t["table"][where], t["table_host"][where] = value, value
        out, lse = _call(t, flag=1)
        _check(t, out, lse)
    # none at all: zeros and -inf
    t = dict(s, table=torch.full_like(s["table"], -1), table_host=np.full_like(s["table_host"], -1))
    out, lse = _call(t, flag=1)
    assert (out == 0).all() and (lse == -math.inf).all()


def test_a_length_beyond_the_pages_of_a_row():
    s = _make([20, 60], [4, 3], 4, 2, 64, 16, BF)                  # 4 pages of 16 a row: 64 tokens
    t = dict(s, len=s["len"].clone(), lens=[24, 70])
    t["len"][1] = 70                                               # nodes at 67 .. 69: not there; the context up to 63 is
    out, lse = _call(t, flag=1)
    _check(t, out, lse)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("window", [0, 60])
def test_values_that_are_no_numbers_where_a_node_does_not_look(dtype, value, window):
    """Behind the length, in pages of nobody, in brothers and, with a window, in front of it; both of keys and values."""
    s = _make([150, 90], [40, 3], 14, 2, 128, 16, dtype, "tree", seed=3)
    want = _call(s, window=window)
    page, table = 16, s["table_host"]
    for x in (s["k"], s["v"]):
        held = torch.zeros(x.shape[1], dtype=torch.bool)
        held[torch.from_numpy(table[table >= 0]).long()] = True
        x[:, ~held.cuda()] = value
        for i, n in enumerate(s["lens"]):
            x[:, table[i, (n - 1) // page], (n - 1) % page + 1:] = value
    got = _call(s, window=window)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # nodes: those that see a spoilt one are spoilt as the formula has it, all others do not notice
    for i, j in ((0, 3), (0, 39), (1, 1)):
        n = s["first"][i + 1] - s["first"][i]
        t = s["lens"][i] - n + j
        for x in (s["k"], s["v"]):
            keep = x[:, table[i, t // page], t % page].clone()
            x[:, table[i, t // page], t % page, 1, 5] = value
            out, lse = _call(s, window=window)
            x[:, table[i, t // page], t % page] = keep
            a = s["first"][i]
            see = [b for b, tokens in enumerate(T.sees(s["lens"][i] - n, s["parent"][a:a + n], window)) if t in tokens]
            blind = torch.ones(out.shape[0], dtype=torch.bool)
            blind[[a + b for b in see]] = False
            assert torch.equal(out[blind.cuda()], want[0][blind.cuda()]) and torch.equal(lse[blind.cuda()], want[1][blind.cuda()])
            assert torch.equal(out[:, :7], want[0][:, :7])         # heads of the other kv head
            if x is s["v"]:
                spoilt = out[[a + b for b in see]][:, 7:, 5]
                assert not torch.isfinite(spoilt).any()
                others = torch.ones(128, dtype=torch.bool)
                others[5] = False
                assert torch.equal(out[..., others.cuda()], want[0][..., others.cuda()])
    if window:
        # tokens of the context that the deepest nodes no longer see
        depth = [len(x) for x in T.sees(0, s["parent"][:40], 0)]
        t = 150 + min(depth) - 1 - window + 1                      # the first that anybody sees
        s["v"][:, table[0, t // page], t % page] = value
        s["k"][:, table[0, t // page], t % page] = value
        out, lse = _call(s, window=window)
        blind = [b for b, x in enumerate(depth) if x > min(depth)]
        assert blind and torch.equal(out[blind], want[0][blind]) and torch.equal(lse[blind], want[1][blind])


def test_fp16_weights_that_count_only_in_sum():
    """12 000 tokens whose weight is e^-14 of another's, with one value of theirs: half of fp16's steps are above them."""
    for gap in (8.0, 11.0, 14.0, 16.0):
        s = _make([12000], [2], 2, 1, 64, 16, HF, "path")
        s["k"].zero_()
        s["v"].fill_(1.0)
        t = 7
        s["k"][0, s["table_host"][0, 0], t] = 0.25
        s["v"][0, s["table_host"][0, 0], t] = 0.0
        s["q"].fill_(1.0)
        scale = gap / (64 * 0.25)
        out, lse = _call(s, scale=scale)
        tail = 12000 * math.exp(-gap)
        want = tail / (1 + tail)                                   # 12 001 tokens and 12 002 less one
        assert (out.double() - want).abs().max() <= 2.0 ** -9 * want + 12002 * 2.0 ** -32 + 12000 ** -1 * want * 2
        assert torch.isfinite(lse).all()


def test_large_scores_do_not_overflow():
    s = _make([500, 20], [33, 4], 4, 2, 128, 16, BF)
    for scale in (50.0, -50.0, 1e30):
        out, lse = _call(s, scale=scale)
        assert torch.isfinite(out).all()
    out, lse = _call(s, scale=1e-30)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_captured_and_replayed_with_other_lengths_and_trees():
    oqm = _lib()
    s = _make([300, 40], [12, 20], 8, 2, 128, 16, BF, extra=4)
    u = _make([25, 500], [20, 7], 8, 2, 128, 16, BF, seed=9, extra=9, width=s["table"].shape[1] + 15)
    assert s["rows"] == u["rows"]
    width = max(s["table"].shape[1], u["table"].shape[1])
    k = torch.zeros(1, max(s["k"].shape[1], u["k"].shape[1]), 16, 2, 128, dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    table = torch.full((2, width), -1, dtype=torch.int32, device="cuda")
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    first, parent = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(36, dtype=torch.int32, device="cuda")
    q, out, lse = torch.zeros_like(s["q"]), torch.zeros_like(s["q"]), torch.zeros(36, 8, device="cuda")
    pool, seqs = oqm.KvPool(k, v), oqm.KvSeqs(table, n)
    ws = torch.empty(oqm.stom_kv_attend_tree_workspace_bytes(pool, seqs, 36, 8), dtype=torch.uint8, device="cuda")

    def fill(a):
        k[:, :a["k"].shape[1]], v[:, :a["v"].shape[1]] = a["k"], a["v"]
        table.fill_(-1)
        table[:, :a["table"].shape[1]] = a["table"]
        n.copy_(a["len"])
        first.copy_(torch.tensor(a["first"]))
        parent.copy_(torch.tensor(a["parent"] + [-1] * (36 - len(a["parent"]))))
        q.copy_(a["q"])
        out.fill_(7.0)
        lse.fill_(7.0)

    def call():
        oqm.stom_kv_attend_tree(pool, seqs, 0, first, q, out, 128 ** -0.5, ws, parent=parent, lse=lse)

    fill(s)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for a in (s, u, s):
        fill(a)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        _check(a, out, lse)


def test_two_streams_with_their_own_workspaces():
    oqm = _lib()
    calls = []
    for seed, had, new in ((0, [3000], [40]), (4, [100, 2000], [3, 30])):
        s = _make(had, new, 28, 4, 128, 50, BF, seed=seed)
        pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"])
        ws = torch.empty(oqm.stom_kv_attend_tree_workspace_bytes(pool, seqs, s["rows"], 28), dtype=torch.uint8, device="cuda")
        first, parent = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (s["first"], s["parent"]))
        calls.append((s, pool, seqs, ws, first, parent, torch.full_like(s["q"], 7.0), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for s, pool, seqs, ws, first, parent, out, stream in calls:
            oqm.stom_kv_attend_tree(pool, seqs, 0, first, s["q"], out, 128 ** -0.5, ws, parent=parent, stream=stream)
    torch.cuda.synchronize()
    for s, *_, out, _ in calls:
        _check(s, out, None)
