"""Decode attention over a paged cache (stom_kv_attend) against softmax attention in 64 bits.

Tolerance of out, element by element, with u the output type's half step (2^-8 bf16, 2^-11 fp16):
    u |out|                       the one rounding of the result
  + mean_w|V| * (2 u^2 + 2^-15)   what the weights are off by: their low 16-bit part is rounded to u of itself (u^2 of
                                  the weight, with a factor 2 for the subtraction), and scores, exponentials and sums in
                                  binary32: a score of magnitude below 32 carries below 2^-24 * 32 * 8 = 2^-16 from its
                                  sum and its scaling, the exponential doubles it at most; tanh of a capped score adds
                                  2 steps of the cap (2 * 32 * 2^-24)
  + 2^-24 (fp16 only)             where the result is subnormal
lse: 2^-15 absolute by the same sum, plus 2^-22 relative.
Scores stay below 32 in magnitude: |q||k| scale of normal vectors, checked on the oracle's side."""
import math

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


def _close(got, want, mag, dtype):
    u = K.HALF_STEP[dtype]
    lim = u * np.abs(want) + mag * (2 * u * u + 2.0 ** -15) + (2.0 ** -24 if dtype is HF else 0.0)
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    bad = np.abs(got - want) > lim
    assert not bad.any(), (int(bad.sum()), float(np.max(np.abs(got - want) / np.maximum(lim, 1e-30))))


def _case(lens, hq, hk, d, page, dtype, cap=0.0, window=0, order="token", layers=1, layer=0, with_lse=True, seed=0,
          scale=None):
    oqm = _lib()
    rng = np.random.default_rng(seed)
    s = K.paged(rng, lens, page, layers, hk, d, dtype, order=order, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    q = (1.5 * torch.randn(len(lens), hq, d, generator=g, device="cuda")).to(dtype)
    out = torch.full_like(q, 7.0)
    lse = torch.full((len(lens), hq), 7.0, device="cuda") if with_lse else None
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"])
    ws = torch.full((oqm.stom_kv_attend_workspace_bytes(pool, seqs, hq) + 64,), 255, dtype=torch.uint8, device="cuda")
    scale = scale or 1.0 / math.sqrt(d)
    oqm.stom_kv_attend(pool, seqs, layer, q, out, scale, ws[:-64], lse=lse, softcap=cap, window=window, dev_flags=flags)
    torch.cuda.synchronize()
    assert (ws[-64:] == 255).all() and flags.item() == 0
    want, wlse, mag = K.attend_rows(s["k"], s["v"], s["table_host"], lens, q, scale, cap, window, layer)
    assert np.abs(wlse[np.isfinite(wlse)]).max(initial=0.0) < 32
    _close(out, want, mag, dtype)
    if with_lse:
        got = lse.double().cpu().numpy()
        empty = ~np.isfinite(wlse)
        assert (got[empty] == -np.inf).all()
        assert (np.abs(got - wlse)[~empty] <= 2.0 ** -15 + 2.0 ** -22 * np.abs(wlse[~empty])).all()
    return s, q, out


@pytest.mark.parametrize("lens,hq,hk,d,page,dtype", [
    ([1], 4, 4, 64, 16, BF),                           # one token
    ([0], 4, 2, 128, 16, BF),                          # nothing at all
    ([15, 16, 17, 0, 1, 33], 8, 2, 64, 16, HF),        # around a tile's end, an empty row between
    ([2500], 28, 4, 128, 50, BF),                      # one stream over the whole device
    ([700, 3, 0, 0, 1201, 50, 51], 28, 4, 128, 50, BF),
    ([333, 64, 129], 16, 2, 128, 1, HF),               # pages of one token
    ([333, 64, 1000], 12, 1, 128, 7, BF),              # 12 query heads on one kv head, odd pages
    ([90, 400], 12, 1, 64, 33, HF),
    ([513, 30], 40, 2, 128, 64, BF),                   # 20 heads: two blocks of them
    ([513, 30], 20, 1, 256, 64, HF),                   # 20 heads at d = 256: three
    ([300, 77, 5], 8, 4, 256, 16, BF),
    ([64], 64, 1, 64, 8, BF),                          # the largest group
    ([5, 9, 2, 0, 31] * 60, 4, 2, 64, 4, BF),          # 300 short rows
    ([1] * 700 + [40] * 35, 2, 1, 64, 16, HF),
    ([0] * 40 + [3] + [0] * 2000 + [700] + [0] * 50, 2, 1, 64, 16, HF),   # long runs of empty rows
    (([0] * 3 + [1]) * 2048, 1, 1, 64, 2, BF),         # as many rows as it takes
])
def test_matches_plain_attention(lens, hq, hk, d, page, dtype):
    _case(lens, hq, hk, d, page, dtype)


@pytest.mark.parametrize("window", [1, 15, 16, 17, 100, 5000])
def test_window(window):
    _case([1000, 3, 0, 16, 257], 8, 2, 128, 50, BF, window=window)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HF, 64), (BF, 256)])
def test_capped_scores(dtype, d):
    _case([700, 31], 8, 4, d, 16, dtype, cap=3.0, window=300)


def test_head_outer_pages_later_layer_and_no_lse():
    _case([130, 999], 14, 2, 128, 25, BF, order="head", layers=3, layer=2, with_lse=False)


def test_strided_query_output_and_table():
    oqm = _lib()
    rng = np.random.default_rng(5)
    lens, hq, hk, d = [77, 200, 3], 6, 2, 64
    s = K.paged(rng, lens, 16, 1, hk, d, HF, seed=5)
    qkv = torch.randn(3, hq + 2 * hk, d, device="cuda").to(HF)       # q as a slice of a fused projection
    q = qkv[:, :hq]
    big = torch.full((3, 2 * hq, d + 8), 9.0, device="cuda", dtype=HF)
    out = big[:, ::2, :d]
    table = torch.full((3, s["table"].shape[1] + 5), 10 ** 6, dtype=torch.int32, device="cuda")
    table[:, :s["table"].shape[1]] = s["table"]
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(table[:, :s["table"].shape[1]], s["len"])
    ws = torch.empty(oqm.stom_kv_attend_workspace_bytes(pool, seqs, hq), dtype=torch.uint8, device="cuda")
    oqm.stom_kv_attend(pool, seqs, 0, q, out, 0.125, ws)
    want, _, mag = K.attend_rows(s["k"], s["v"], s["table_host"], lens, q, 0.125)
    _close(out, want, mag, HF)
    assert (big[:, 1::2] == 9.0).all() and (big[:, :, d:] == 9.0).all()      # what is not the output stays


def test_bad_pages_count_as_absent_and_long_rows_are_cut():
    oqm = _lib()
    rng = np.random.default_rng(6)
    lens, hq, hk, d = [100, 64, 40], 4, 2, 64
    s = K.paged(rng, lens, 16, 1, hk, d, BF, seed=6)
    table = s["table_host"].copy()
    table[0, 2], table[1, 3], table[2, :3] = -1, s["k"].shape[1], 1 << 30
    dev = torch.from_numpy(table).cuda()
    length = torch.tensor([10 ** 6, 64, 40], dtype=torch.int32, device="cuda")       # the first beyond its pages
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.randn(3, hq, d, device="cuda").to(BF)
    out, lse = torch.empty_like(q), torch.empty(3, hq, device="cuda")
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(dev, length)
    ws = torch.empty(oqm.stom_kv_attend_workspace_bytes(pool, seqs, hq), dtype=torch.uint8, device="cuda")
    oqm.stom_kv_attend(pool, seqs, 0, q, out, 0.125, ws, lse=lse, dev_flags=flags)
    want, wlse, mag = K.attend_rows(s["k"], s["v"], table, length.tolist(), q, 0.125)
    _close(out, want, mag, BF)
    assert flags.item() & oqm.FLAG_BAD_INDEX
    assert (lse[2] == -math.inf).all() and (out[2] == 0).all()               # all of its pages are bad


def test_nothing_behind_the_length_is_read():
    oqm = _lib()
    rng = np.random.default_rng(7)
    lens = [33, 50, 1]
    s = K.paged(rng, lens, 50, 1, 2, 128, BF, seed=7)
    q = torch.randn(3, 4, 128, device="cuda").to(BF)
    want, _, mag = K.attend_rows(s["k"], s["v"], s["table_host"], lens, q, 0.1)
    for i, n in enumerate(lens):                                             # poison what is not in use
        page = s["table_host"][i, 0]
        s["k"][:, page, n:] = math.nan
        s["v"][:, page, n:] = math.inf
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"])
    ws = torch.empty(oqm.stom_kv_attend_workspace_bytes(pool, seqs, 4), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    oqm.stom_kv_attend(pool, seqs, 0, q, out, 0.1, ws)
    _close(out, want, mag, BF)


def test_offsets_beyond_32_bits():
    """Pages so far apart that an element's offset passes 2^31 and its byte offset 2^33."""
    oqm = _lib()
    stride = 1 << 26                                                          # elements between pages
    k = torch.empty(1, 72, stride, dtype=HF, device="cuda")[:, :, :16 * 64].view(1, 72, 16, 1, 64)
    v = torch.empty_strided(k.shape, k.stride(), dtype=HF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    k.copy_(torch.randn(k.shape, generator=g, device="cuda"))
    v.copy_(torch.randn(k.shape, generator=g, device="cuda"))
    assert k.stride(1) * 71 > 1 << 32
    table = np.array([[71, 0, 40, 70]], np.int32)
    q = torch.randn(1, 4, 64, device="cuda").to(HF)
    out = torch.empty_like(q)
    pool = oqm.KvPool(k, v)
    seqs = oqm.KvSeqs(torch.from_numpy(table).cuda(), torch.tensor([61], dtype=torch.int32, device="cuda"))
    ws = torch.empty(oqm.stom_kv_attend_workspace_bytes(pool, seqs, 4), dtype=torch.uint8, device="cuda")
    oqm.stom_kv_attend(pool, seqs, 0, q, out, 0.125, ws)
    want, _, mag = K.attend_rows(k, v, table, [61], q, 0.125)
    _close(out, want, mag, HF)


def test_same_result_every_time_and_two_graphs_share_a_workspace():
    oqm = _lib()
    rng = np.random.default_rng(8)
    lens = [5000, 3, 777]
    s = K.paged(rng, lens, 50, 2, 4, 128, BF, seed=8)
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"])
    ws = torch.empty(oqm.stom_kv_attend_workspace_bytes(pool, seqs, 28), dtype=torch.uint8, device="cuda")
    qs = [torch.randn(3, 28, 128, device="cuda").to(BF) for _ in range(2)]
    eager = []
    for layer in range(2):
        o = torch.empty_like(qs[layer])
        oqm.stom_kv_attend(pool, seqs, layer, qs[layer], o, 0.09, ws)
        eager.append(o)
    side = torch.cuda.Stream()
    graphs, outs = [], []
    for layer in range(2):
        o = torch.zeros_like(qs[layer])
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            oqm.stom_kv_attend(pool, seqs, layer, qs[layer], o, 0.09, ws)
        graphs.append(g)
        outs.append(o)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for o, e in zip(outs, eager):
        assert torch.equal(o, e)
    # the lengths are read from the device: a captured step follows them
    s["len"].copy_(torch.tensor([20, 0, 700], dtype=torch.int32))
    graphs[0].replay()
    torch.cuda.synchronize()
    want, _, mag = K.attend_rows(s["k"], s["v"], s["table_host"], [20, 0, 700], qs[0], 0.09)
    _close(outs[0], want, mag, BF)


def test_on_another_stream():
    oqm = _lib()
    rng = np.random.default_rng(9)
    s = K.paged(rng, [400, 90], 16, 1, 2, 64, BF, seed=9)
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"])
    q = torch.randn(2, 4, 64, device="cuda").to(BF)
    outs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for st in streams:                                                       # two calls at once, a workspace each
        ws = torch.empty(oqm.stom_kv_attend_workspace_bytes(pool, seqs, 4), dtype=torch.uint8, device="cuda")
        o = torch.empty_like(q)
        torch.cuda.synchronize()
        oqm.stom_kv_attend(pool, seqs, 0, q, o, 0.125, ws, stream=st)
        outs.append((o, ws))
    torch.cuda.synchronize()
    want, _, mag = K.attend_rows(s["k"], s["v"], s["table_host"], [400, 90], q, 0.125)
    for o, _ in outs:
        _close(o, want, mag, BF)


def _sink_row(lens, gap, hq, hk, d, page, dtype, at=0, seed=0):
    """One token of every row stands `gap` nats above all others, whose scores are zero, and has a value of zero; all other
    values are positive.  The result is the tail's alone, however little a token of it weighs."""
    oqm = _lib()
    s = K.paged(np.random.default_rng(seed), lens, page, 1, hk, d, dtype, seed=seed)
    s["k"].zero_()
    s["v"].copy_(s["v"].abs() + 0.25)
    for i, n in enumerate(lens):
        if n:
            t = min(at, n - 1)
            s["k"][0, s["table_host"][i, t // page], t % page, :, 0] = gap
            s["v"][0, s["table_host"][i, t // page], t % page] = 0
    q = torch.zeros(len(lens), hq, d, dtype=dtype, device="cuda")
    q[:, :, 0] = 4.0                                     # 4 * gap * 0.25: the score is exact
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"])
    ws = torch.full((oqm.stom_kv_attend_workspace_bytes(pool, seqs, hq),), 255, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((len(lens), hq), 7.0, device="cuda")
    oqm.stom_kv_attend(pool, seqs, 0, q, out, 0.25, ws, lse=lse)
    want, wlse, mag = K.attend_rows(s["k"], s["v"], s["table_host"], lens, q, 0.25)
    _close(out, want, mag, dtype)
    some = np.isfinite(wlse)
    assert (np.abs(lse.double().cpu().numpy() - wlse)[some] <= 2.0 ** -15 + 2.0 ** -22 * np.abs(wlse[some])).all()


@pytest.mark.parametrize("gap", [10.0, 13.0, 15.0, 15.5, 17.0, 17.5])
@pytest.mark.parametrize("lens,hq,hk,d,page", [
    ([48, 33, 0, 90] * 700, 1, 1, 64, 16),               # units that a warp holds whole
    ([600] * 300, 2, 1, 64, 50),                         # units of several warps of a block
    ([12583], 2, 1, 128, 50),                            # one unit over all blocks
    ([5000, 40], 12, 1, 128, 7),                         # 16 heads a product
    ([3000, 17], 1, 1, 256, 16),
])
def test_a_tail_that_counts_only_in_sum(lens, hq, hk, d, page, gap):
    """fp16: a tail's weights are far below the type's smallest steps relative to the row's largest.  _close's limit has
    room: a weight's two parts are off by 2^-22 of themselves or by 2^-40 of the largest weight of their 16 tokens,
    whichever is more, and in the sum over the 15 tokens beside the sink that is below 2^-36, against the limit's 2^-24."""
    _sink_row(lens, gap, hq, hk, d, page, HF, at=3)


@pytest.mark.parametrize("n,gap", [(131072, 20.0), (131072, 24.0), (400009, 22.5)])
def test_a_long_tail_that_counts_only_in_sum(n, gap):
    _sink_row([n], gap, 1, 1, 64, 64, HF, at=n // 2)


def test_a_tail_in_bf16():
    _sink_row([12583, 600, 40], 17.0, 2, 1, 128, 50, BF, at=3)


@pytest.mark.parametrize("window", [0, 1, 20, 40, 64, 100, 5000])
def test_lengths_beyond_the_pages_of_a_row(window):
    """All pages are good: what a length has beyond them is absent, and flagged.  A window ends at the length, so it may
    reach behind the pages in part or as a whole."""
    oqm = _lib()
    room, hq, hk, d = 64, 4, 2, 64
    s = K.paged(np.random.default_rng(11), [room] * 5, 16, 1, hk, d, BF, seed=11)
    lens = [100, 64, 70, 2 ** 31 - 1, 9]
    q = torch.randn(5, hq, d, device="cuda").to(BF)
    pool = oqm.KvPool(s["k"], s["v"])
    for rows, flag in ((slice(0, 5), oqm.FLAG_BAD_INDEX), (slice(1, 2), 0), (slice(4, 5), 0), (slice(2, 3), oqm.FLAG_BAD_INDEX)):
        n = torch.tensor(lens[rows], dtype=torch.int32, device="cuda")
        seqs = oqm.KvSeqs(s["table"][rows], n)
        ws = torch.empty(oqm.stom_kv_attend_workspace_bytes(pool, seqs, hq), dtype=torch.uint8, device="cuda")
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = torch.full_like(q[rows], 7.0), torch.full((len(n), hq), 7.0, device="cuda")
        oqm.stom_kv_attend(pool, seqs, 0, q[rows], out, 0.125, ws, lse=lse, window=window, dev_flags=flags)
        torch.cuda.synchronize()
        assert flags.item() == flag
        for j, length in enumerate(lens[rows]):
            i = rows.start + j
            end = min(length, room)
            seen = end - (max(0, length - window) if window else 0)           # tokens of the window that are there
            if seen <= 0:
                assert (out[j] == 0).all() and (lse[j] == -math.inf).all()
                continue
            want, wlse, mag = K.attend_rows(s["k"], s["v"], s["table_host"][i:i + 1], [end], q[i:i + 1], 0.125, window=seen)
            _close(out[j:j + 1], want, mag, BF)
            assert (np.abs(lse[j].double().cpu().numpy() - wlse[0]) <= 2.0 ** -15 + 2.0 ** -22 * np.abs(wlse[0])).all()
