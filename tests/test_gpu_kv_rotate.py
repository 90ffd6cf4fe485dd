"""Rotary positions and per-head norms (stom_kv_rotate, stom_kv_append) against the formulas in 64 bits.

Tolerance, element by element, u the type's half step:
    u |out|              the one rounding
  + 2^-20 mag            mag = |a| + |b| of the turned pair (or |y|): binary32 sine and cosine of an angle reduced in
                         binary64 (within 2 ulp, 2^-22 of 1; the angle itself is off by at most 2^-52 of |pos freq| <= 2^21,
                         2^-31), three roundings of the turn (3 * 2^-24), and of the norm the sum of d <= 256 squares
                         (relative 2^-24 * 17 by its tree of 16 adds a thread and 4 exchanges, halved by the root),
                         division, root and two products (2^-22): together below 2^-20
  + 2^-24 (fp16 only)    where the result is subnormal"""
import numpy as np
import pytest
import torch

import _kv as K

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def _lib():
    from paper_2510_18269_b200 import oqm
    oqm.lib()
    return oqm


def _close(got, want, mag, dtype):
    lim = K.HALF_STEP[dtype] * np.abs(want) + 2.0 ** -20 * mag + (2.0 ** -24 if dtype is HF else 0.0)
    d = np.abs(got.double().cpu().numpy() - want)
    assert (d <= lim).all(), (int((d > lim).sum()), float(np.max(d / np.maximum(lim, 1e-30))))


def _rope(oqm, rot, layout, magnitude=1.0, **kw):
    return oqm.Rope(oqm.stom_kv_frequencies(rot, **kw).cuda() if rot else None, layout=layout, magnitude=magnitude)


def _freq(rope):
    return rope.freq if rope.freq is not None else torch.zeros(0, dtype=torch.float64)


@pytest.mark.parametrize("n,hq,hk,d,rot,layout,norm,dtype", [
    (1, 28, 4, 128, 128, 0, False, BF),
    (1, 1, 1, 64, 16, 1, True, HF),
    (7, 16, 8, 64, 64, 1, True, FL),
    (33, 5, 3, 128, 64, 0, True, BF),                  # odd head counts, half of a head
    (33, 5, 3, 128, 48, 1, True, HF),
    (3, 40, 1, 256, 256, 0, False, FL),
    (3, 40, 1, 256, 16, 0, True, BF),
    (50, 4, 2, 64, 0, 0, True, BF),                    # norms alone
    (50, 4, 2, 64, 0, 0, False, BF),                   # a copy
    (2500, 3, 2, 64, 32, 0, True, HF),                 # four tokens a block, the last block not full
    (2401, 2, 1, 128, 128, 1, False, FL),
])
def test_rotate(n, hq, hk, d, rot, layout, norm, dtype):
    oqm = _lib()
    g = torch.Generator(device="cuda").manual_seed(n + d + rot)
    q, k = ((3 * torch.randn(n, h, d, generator=g, device="cuda")).to(dtype) for h in (hq, hk))
    pos = torch.randint(0, 1 << 21, (n,), generator=g, device="cuda").to(torch.int32)
    qw, kw = ((1 + 0.3 * torch.randn(d, generator=g, device="cuda")) if norm else None for _ in range(2))
    rope = _rope(oqm, rot, layout, magnitude=1.25)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    oqm.stom_kv_rotate(rope, pos, q=q, q_out=qo, k=k, k_out=ko, q_weight=qw, k_weight=kw)
    torch.cuda.synchronize()
    for x, o, w in ((q, qo, qw), (k, ko, kw)):
        want, mag = K.turned(x, pos, _freq(rope), layout, w, magnitude=1.25)
        _close(o, want, mag, dtype)
    if not norm and not rot:
        assert torch.equal(q, qo)
    # in place, queries and keys apart: the same bits
    q2, k2 = q.clone(), k.clone()
    oqm.stom_kv_rotate(rope, pos, q=q2, q_out=q2, q_weight=qw)
    oqm.stom_kv_rotate(rope, pos, k=k2, k_out=k2, k_weight=kw)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


def test_norm_of_queries_only_and_zero_rows():
    oqm = _lib()
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k = torch.randn(9, 4, 64, generator=g, device="cuda").to(BF), torch.randn(9, 2, 64, generator=g, device="cuda").to(BF)
    q[3] = 0
    w = torch.rand(64, generator=g, device="cuda")
    pos = torch.arange(9, dtype=torch.int32, device="cuda") - 4                   # negative positions turn backwards
    rope = _rope(oqm, 64, 0)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    oqm.stom_kv_rotate(rope, pos, q=q, q_out=qo, k=k, k_out=ko, q_weight=w, eps=1e-5)
    want, mag = K.turned(q, pos, rope.freq, 0, w, eps=1e-5)
    _close(qo, want, mag, BF)
    want, mag = K.turned(k, pos, rope.freq, 0)
    _close(ko, want, mag, BF)
    assert (qo[3] == 0).all()


def test_slices_of_a_fused_projection_and_guards():
    oqm = _lib()
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(21, 8 + 2 + 2, 128, generator=g, device="cuda").to(HF)
    q, k = x[:, :8], x[:, 8:10]
    big = torch.full((21, 12, 136), 5.0, device="cuda", dtype=HF)
    pos = torch.arange(21, dtype=torch.int32, device="cuda") * 1000
    rope = _rope(oqm, 128, 1)
    oqm.stom_kv_rotate(rope, pos, q=q, q_out=big[:, 0:8, :128], k=k, k_out=big[:, 9:11, :128])
    want, mag = K.turned(q, pos, rope.freq, 1)
    _close(big[:, :8, :128], want, mag, HF)
    want, mag = K.turned(k, pos, rope.freq, 1)
    _close(big[:, 9:11, :128], want, mag, HF)
    assert (big[:, 8] == 5).all() and (big[:, 11] == 5).all() and (big[..., 128:] == 5).all()


def test_scaled_frequencies_reach_the_kernel():
    oqm = _lib()
    q = torch.randn(40, 2, 64, device="cuda")
    pos = torch.arange(40, dtype=torch.int32, device="cuda") * 20000
    for kw in (dict(scaling=oqm.ROPE_LINEAR, factor=4.0), dict(scaling=oqm.ROPE_BASE, factor=8.0),
               dict(scaling=oqm.ROPE_WAVES, factor=8.0, trained=8192.0)):
        rope = _rope(oqm, 64, 0, **kw)
        o = torch.empty_like(q)
        oqm.stom_kv_rotate(rope, pos, q=q, q_out=o)
        want, mag = K.turned(q, pos, oqm.stom_kv_frequencies(64, **kw), 0)
        _close(o, want, mag, FL)


def _append(hq, hk, d, page, dtype, norm, order, with_q, decode, seed):
    oqm = _lib()
    rng = np.random.default_rng(seed)
    lens = [70, 1, 200, 49, 51]
    s = K.paged(rng, lens, page, 2, hk, d, dtype, order=order, seed=seed)
    before_k, before_v = s["k"].clone(), s["v"].clone()
    if decode:
        seq, slot = None, np.array(lens) - 1
        who = np.arange(len(lens))
    else:
        who = np.repeat(np.arange(len(lens)), [20, 1, 33, 2, 50])
        slot = np.concatenate([np.arange(n - c, n) for n, c in zip(lens, [20, 1, 33, 2, 50])])
        mix = rng.permutation(len(who))                                          # tokens in any order
        who, slot = who[mix], slot[mix]
        seq = torch.from_numpy(who.astype(np.int32)).cuda()
        slot[3] = slot[40] = -1                                                  # padding
    n = len(slot)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v = (torch.randn(n, h, d, generator=g, device="cuda").to(dtype) for h in (hq, hk, hk))
    pos = torch.from_numpy((np.maximum(slot, 0) + 1000).astype(np.int32)).cuda()
    w = 1 + 0.3 * torch.randn(d, generator=g, device="cuda") if norm else None
    rope = _rope(oqm, d // 2, 0)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    qo = torch.full_like(q, 3.0)
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"], s["refs"])
    oqm.stom_kv_append(pool, seqs, 1, rope, pos, torch.from_numpy(slot.astype(np.int32)).cuda(), k, v,
                       q=q if with_q else None, q_out=qo if with_q else None, seq=seq, q_weight=w if with_q else None,
                       k_weight=w, dev_flags=flags)
    torch.cuda.synchronize()
    assert flags.item() == 0
    wk, mk = K.turned(k, pos, rope.freq, 0, w)
    if with_q:
        want, mag = K.turned(q, pos, rope.freq, 0, w)
        _close(qo, want, mag, dtype)
    else:
        assert (qo == 3).all()
    kept = slot >= 0
    pid = s["table_host"][who[kept], slot[kept] // page]
    off = slot[kept] % page
    _close(s["k"][1, pid, off], wk[kept], mk[kept], dtype)
    assert torch.equal(s["v"][1, pid, off], v[torch.from_numpy(kept).cuda()])
    before_k[1, pid, off], before_v[1, pid, off] = s["k"][1, pid, off], s["v"][1, pid, off]
    assert torch.equal(before_k, s["k"]) and torch.equal(before_v, s["v"])       # nothing else was written


@pytest.mark.parametrize("hq,hk,d,page,dtype,norm,order,with_q,decode", [
    (28, 4, 128, 50, BF, False, "token", True, True),
    (8, 2, 64, 7, HF, True, "head", True, False),
    (3, 1, 256, 16, BF, True, "token", True, False),
    (4, 4, 64, 1, HF, False, "token", False, False),
    (40, 8, 128, 64, BF, True, "head", True, True),
])
def test_append(hq, hk, d, page, dtype, norm, order, with_q, decode):
    _append(hq, hk, d, page, dtype, norm, order, with_q, decode, seed=hq + d)


def test_append_skips_and_flags_what_has_no_place():
    oqm = _lib()
    rng = np.random.default_rng(4)
    s = K.paged(rng, [40, 40], 16, 1, 2, 64, BF, seed=4)
    s["table"][1, 1] = 10 ** 6
    before = s["k"].clone()
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"])
    k = torch.randn(6, 2, 64, device="cuda").to(BF)
    q, qo = torch.randn(6, 2, 64, device="cuda").to(BF), torch.zeros(6, 2, 64, device="cuda", dtype=BF)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    rope = _rope(oqm, 0, 0)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    # beyond the row, a page that is none, a sequence that is none (two), a negative slot that is not padding, and one good
    oqm.stom_kv_append(pool, seqs, 0, rope, i32(*range(6)), i32(48, 20, 0, 0, -2, 39), k, k, q=q, q_out=qo,
                       seq=i32(0, 1, 2, -1, 0, 0), dev_flags=flags)
    assert flags.item() == oqm.FLAG_BAD_INDEX and torch.equal(q, qo)
    page = int(s["table_host"][0, 2])
    assert torch.equal(s["k"][0, page, 7], k[5])
    before[0, page, 7] = k[5]
    assert torch.equal(before, s["k"])


def test_replayed_decode_step():
    oqm = _lib()
    rng = np.random.default_rng(6)
    s = K.paged(rng, [60, 60], 16, 1, 2, 64, BF, seed=6)
    pool, seqs = oqm.KvPool(s["k"], s["v"]), oqm.KvSeqs(s["table"], s["len"])
    rope = _rope(oqm, 64, 0)
    q, k, v = (torch.randn(2, h, 64, device="cuda").to(BF) for h in (4, 2, 2))
    qo = torch.empty_like(q)
    at = torch.tensor([10, 20], dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        oqm.stom_kv_append(pool, seqs, 0, rope, at, at, k, v, q=q, q_out=qo)
    for step in range(3):
        q.copy_(torch.randn_like(q.float()))
        k.copy_(torch.randn_like(k.float()))
        at += 1
        g.replay()
        torch.cuda.synchronize()
        want, mag = K.turned(q, at, rope.freq, 0)
        _close(qo, want, mag, BF)
        want, mag = K.turned(k, at, rope.freq, 0)
        slot = at.cpu().numpy()
        _close(s["k"][0, s["table_host"][[0, 1], slot // 16], slot % 16], want, mag, BF)
