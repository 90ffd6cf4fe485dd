"""The answering side as it is used, one call after another: groups retrieved from the quantized bank straight into a
stream's pages, their keys rotated in place, then decode steps -- reserve, append, attend in every layer, choose a token
-- for two candidate answers that share the retrieved pages, one of them dropped, the pages moved together.  Every stage
is compared with the plain implementation on what the stages before it left."""
import math

import numpy as np
import pytest
import torch

import _kv as K
import _parity as P
from paper_2510_18269_b200 import synth
from test_gpu_kv_attend import _close as close_attend
from test_gpu_kv_rotate import _close as close_rotate

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
L, HQ, HK, D, G, T, TQ, TOPK, N_SEQS, PAGES = 2, 28, 4, 128, 50, 40, 4, 6, 3, 24
VOCAB = 5003


class Stream:
    def __init__(self, orc):
        from paper_2510_18269_b200 import oqm
        oqm.lib()
        self.oqm = oqm
        sh = synth.Shape("answer", L=L, H_q=HQ, H_k=HK, d=D, G=G, T=T, T_q=TQ, k=TOPK, seed=11)
        _, gcfg, _, bank, _ = P.random_bank(orc, oqm, sh, 0, seed=5)
        dev = dict(device="cuda")
        self.k = torch.full((L, PAGES, G, HK, D), 9.0, dtype=BF, **dev)
        self.v = torch.full_like(self.k, 9.0)
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, **dev)  # noqa: E731
        self.table = torch.full((N_SEQS, 10), -1, dtype=torch.int32, **dev)
        self.len, self.refs, self.flags = i32(N_SEQS), i32(PAGES), i32(1)
        self.pool, self.seqs = oqm.KvPool(self.k, self.v), oqm.KvSeqs(self.table, self.len, self.refs)
        self.pages_ws = torch.empty(oqm.stom_kv_pages_workspace_bytes(self.pool, self.seqs), dtype=torch.uint8, **dev)
        self.attend_ws = torch.empty(oqm.stom_kv_attend_workspace_bytes(self.pool, self.seqs, HQ), dtype=torch.uint8, **dev)
        self.rope = oqm.Rope(oqm.stom_kv_frequencies(D).cuda(), layout=oqm.ROPE_HALF)

        # the retrieved groups go to sequence 0: an empty pool gives pages 0, 1, 2, ..., one contiguous token axis
        self.grow([TOPK * G, 0, 0])
        assert self.table[0, :TOPK].tolist() == list(range(TOPK))
        Q = synth.queries(sh).cuda()
        scores, idx = torch.empty(L, T, **dev), i32(L, TOPK)
        ws = torch.empty(oqm.stom_oqm_retrieve_workspace_bytes(gcfg, L, T, TOPK), dtype=torch.uint8, **dev)
        strides = (self.k.stride(0), self.k.stride(3), self.k.stride(2))
        oqm.stom_oqm_retrieve(gcfg, bank, 0, L, T, Q, TQ, P.q_strides(sh), TOPK, scores, idx, self.k, self.v, oqm.BF16,
                              strides, 0, ws, dev_flags=self.flags)
        # the same groups into a cache of the usual layout
        ka, va = (torch.zeros(L, HK, TOPK * G, D, dtype=BF, **dev) for _ in range(2))
        oqm.stom_oqm_dequant_gather(gcfg, bank, 0, L, idx, TOPK, T, ka, va, oqm.BF16, ka.stride()[:3], 0)
        for x, y in ((self.k, ka), (self.v, va)):
            assert torch.equal(x[:, :TOPK].reshape(L, TOPK * G, HK, D), y.permute(0, 2, 1, 3))
            assert (x[:, TOPK:] == 9.0).all()
        # stored keys were not rotated: all layers in one call, in place
        keys = self.k[:, :TOPK].reshape(L, TOPK * G, HK, D).clone()     # as they were
        pos = torch.arange(TOPK * G, dtype=torch.int32, **dev)
        for l in range(L):
            rows = self.k[l].view(PAGES * G, HK, D)[:TOPK * G]
            oqm.stom_kv_rotate(self.rope, pos, k=rows, k_out=rows)
            want, mag = K.turned(keys[l], pos, self.rope.freq, 0)
            close_rotate(rows, want, mag, BF)

        g = torch.Generator(device="cuda").manual_seed(3)
        self.rand = lambda *s: torch.randn(*s, generator=g, **dev)  # noqa: E731
        self.head = self.rand(HQ * D, VOCAB) * 0.2
        # what a step works in: filled anew before every step, so that a captured step can be replayed
        self.q, self.kn, self.vn = self.rand(L, N_SEQS, HQ, D).to(BF), self.rand(L, N_SEQS, HK, D).to(BF), self.rand(L, N_SEQS, HK, D).to(BF)
        self.qr, self.out = torch.empty_like(self.q), torch.zeros_like(self.q)
        self.lse = torch.empty(N_SEQS, HQ, **dev)
        self.logits = torch.empty(N_SEQS, VOCAB, **dev)
        self.want, self.slot, self.u = i32(N_SEQS), i32(N_SEQS), torch.zeros(N_SEQS, **dev)
        self.token, self.kept = i32(N_SEQS), i32(N_SEQS)
        self.top_p = torch.full((N_SEQS,), 0.8, **dev)

    def grow(self, want):
        self.oqm.stom_kv_reserve(self.pool, self.seqs, torch.tensor(want, dtype=torch.int32, device="cuda"), self.pages_ws,
                                 dev_flags=self.flags)

    def fill(self, seed):
        """New projections and random numbers, and the lengths to come: every live sequence gets one token."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        for x in (self.q, self.kn, self.vn):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        self.u.copy_(torch.rand(N_SEQS, generator=g, device="cuda"))
        live = self.len > 0
        self.want.copy_(torch.where(live, self.len + 1, 0))
        self.slot.copy_(torch.where(live, self.len, -1))         # -1: nothing to store

    def step(self):
        o = self.oqm
        o.stom_kv_reserve(self.pool, self.seqs, self.want, self.pages_ws, dev_flags=self.flags)
        for l in range(L):
            o.stom_kv_append(self.pool, self.seqs, l, self.rope, self.slot, self.slot, self.kn[l], self.vn[l], q=self.q[l],
                             q_out=self.qr[l], dev_flags=self.flags)
            o.stom_kv_attend(self.pool, self.seqs, l, self.qr[l], self.out[l], 1 / math.sqrt(D), self.attend_ws, lse=self.lse,
                             dev_flags=self.flags)
        torch.matmul(self.out[-1].reshape(N_SEQS, HQ * D).float(), self.head, out=self.logits)
        o.stom_sample_tokens(self.logits, self.u, self.token, top_p=self.top_p, kept=self.kept, dev_flags=self.flags)

    def check(self):
        torch.cuda.synchronize()
        assert self.flags.item() == 0
        lens, table = self.len.tolist(), self.table.cpu().numpy()
        for l in range(L):
            want, mag = K.turned(self.q[l], self.slot, self.rope.freq, 0)
            close_rotate(self.qr[l], want, mag, BF)
            keys, kmag = K.turned(self.kn[l], self.slot, self.rope.freq, 0)
            for i, n in enumerate(lens):
                if n:
                    page, off = table[i, (n - 1) // G], (n - 1) % G
                    close_rotate(self.k[l, page, off], keys[i], kmag[i], BF)
                    assert torch.equal(self.v[l, page, off], self.vn[l, i])
            want, lse, mag = K.attend_rows(self.k, self.v, table, lens, self.qr[l], 1 / math.sqrt(D), layer=l)
            close_attend(self.out[l], want, mag, BF)
        rows = self.logits.double().cpu().numpy()
        for i in range(N_SEQS):
            tokens, counts, _ = K.choose(rows[i], float(self.u[i]), top_p=float(self.top_p[i]))
            assert int(self.token[i]) in tokens and int(self.kept[i]) in counts


def test_answering(orc):
    s = Stream(orc)
    s.fill(1)
    s.step()
    s.check()
    assert s.len.tolist() == [TOPK * G + 1, 0, 0]
    # two candidates share all pages; the step after copies the partly filled last page for one of them
    s.oqm.stom_kv_fork(s.pool, s.seqs, torch.tensor([-1, 0, 0], dtype=torch.int32, device="cuda"), dev_flags=s.flags)
    assert s.refs[:TOPK].tolist() == [3] * TOPK
    for seed in range(2, 5):
        s.fill(seed)
        s.step()
        s.check()
    assert len(set(s.table[:, TOPK].tolist())) == 3
    # the stream itself ends; the pages of the candidates move to the front of the pool and give the same result
    s.oqm.stom_kv_free(s.pool, s.seqs, torch.tensor([1, 0, 0], dtype=torch.int32, device="cuda"), dev_flags=s.flags)
    live = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = torch.empty_like(s.out[0])
    s.oqm.stom_kv_attend(s.pool, s.seqs, 0, s.qr[0], before, 0.1, s.attend_ws)
    s.oqm.stom_kv_compact(s.pool, s.seqs, s.table, s.refs, live, s.pages_ws, dev_flags=s.flags)
    after = torch.empty_like(before)
    s.oqm.stom_kv_attend(s.pool, s.seqs, 0, s.qr[0], after, 0.1, s.attend_ws)
    assert live.item() == TOPK + 2 and int((s.refs > 0).sum()) == TOPK + 2 and (s.refs[TOPK + 2:] == 0).all()
    assert torch.equal(before, after) and (after[0] == 0).all()
    s.fill(9)
    s.step()
    s.check()


def test_captured_decode_step(orc):
    """A whole step as one graph: lengths, pages and tokens come from the device, so it is replayed as it is."""
    s = Stream(orc)
    s.oqm.stom_kv_fork(s.pool, s.seqs, torch.tensor([-1, 0, -1], dtype=torch.int32, device="cuda"), dev_flags=s.flags)
    s.fill(1)
    s.step()                                                      # libraries load outside of the capture
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.step()
    for seed in range(2, 2 + G + 2):                              # over the end of a page
        s.fill(seed)
        g.replay()
        if seed < 4 or seed > G:
            s.check()
    assert s.len.tolist()[:2] == [TOPK * G + G + 3] * 2


def test_an_empty_batch_changes_nothing():
    """No token, no sequence, no row: every call returns, and only the pool's counts are looked at."""
    from paper_2510_18269_b200 import oqm
    oqm.lib()

    def i32(*shape):
        return torch.zeros(*shape, dtype=torch.int32, device="cuda")

    k = torch.randn(1, 6, 16, 2, 64, device="cuda").to(torch.bfloat16)
    pool = oqm.KvPool(k, k.clone())
    before = pool.k.clone(), pool.v.clone()
    refs = i32(6)
    seqs = oqm.KvSeqs(i32(0, 4), i32(0), refs)
    flags = i32(1)
    rope = oqm.Rope(oqm.stom_kv_frequencies(64).cuda())
    q, kv = torch.empty(0, 8, 64, dtype=k.dtype, device="cuda"), torch.empty(0, 2, 64, dtype=k.dtype, device="cuda")
    ws = torch.empty(max(oqm.stom_kv_attend_workspace_bytes(pool, seqs, 8), oqm.stom_kv_pages_workspace_bytes(pool, seqs)),
                     dtype=torch.uint8, device="cuda")
    oqm.stom_kv_reserve(pool, seqs, i32(0), ws, dev_flags=flags)
    oqm.stom_kv_fork(pool, seqs, i32(0), dev_flags=flags)
    oqm.stom_kv_rotate(rope, i32(0), q, q, kv, kv)
    oqm.stom_kv_append(pool, seqs, 0, rope, i32(0), i32(0), kv, kv, q=q, q_out=q, dev_flags=flags)
    oqm.stom_kv_attend(pool, seqs, 0, q, torch.empty_like(q), 0.125, ws, dev_flags=flags)
    oqm.stom_sample_tokens(torch.empty(0, 99, device="cuda"), torch.empty(0, device="cuda"), i32(0), dev_flags=flags)
    oqm.stom_kv_free(pool, seqs, i32(0), dev_flags=flags)
    live = i32(1) + 7
    refs[4] = 1                                                  # a page that no row of these holds
    pool.k[:, 4] = pool.v[:, 4] = before[0][:, 0] = before[1][:, 0] = 1.0
    oqm.stom_kv_compact(pool, seqs, i32(0, 4), refs, live, ws, dev_flags=flags)
    assert live.item() == 1 and refs.tolist() == [1, 0, 0, 0, 0, 0] and flags.item() == 0
    for got, want in ((pool.k, before[0]), (pool.v, before[1])):
        want[:, 4] = 1.0                                         # what stood there stays
        assert torch.equal(got, want)


def test_a_step_that_finds_no_page_writes_nothing():
    """As in a captured step, where nobody looks between the calls: the token of a row whose page is not there is left
    out, and so is what it would have overwritten."""
    from paper_2510_18269_b200 import oqm
    oqm.lib()
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    k = torch.randn(1, 3, 16, 2, 64, device="cuda").to(BF)
    pool = oqm.KvPool(k, k.clone())
    table, n, refs, flags = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), i32(0, 0), i32(0, 0, 0), i32(0)
    seqs = oqm.KvSeqs(table, n, refs)
    ws = torch.empty(max(oqm.stom_kv_pages_workspace_bytes(pool, seqs), oqm.stom_kv_attend_workspace_bytes(pool, seqs, 2)),
                     dtype=torch.uint8, device="cuda")
    oqm.stom_kv_reserve(pool, seqs, i32(32, 16), ws, dev_flags=flags)
    assert flags.item() == 0 and (refs == 1).all()
    before = pool.k.clone(), pool.v.clone(), table.clone()
    q, new = torch.randn(2, 2, 64, device="cuda").to(BF), torch.ones(2, 2, 64, device="cuda", dtype=BF)
    qo, out = torch.empty_like(q), torch.empty_like(q)
    oqm.stom_kv_reserve(pool, seqs, i32(33, 17), ws, dev_flags=flags)
    oqm.stom_kv_append(pool, seqs, 0, oqm.Rope(), i32(32, 16), i32(32, 16), new, new, q=q, q_out=qo, dev_flags=flags)
    oqm.stom_kv_attend(pool, seqs, 0, qo, out, 0.125, ws, dev_flags=flags)
    assert flags.item() == oqm.FLAG_NO_PAGE | oqm.FLAG_BAD_INDEX and n.tolist() == [32, 16]
    assert torch.equal(pool.k, before[0]) and torch.equal(pool.v, before[1]) and torch.equal(table, before[2])
    want, _, mag = K.attend_rows(pool.k, pool.v, table.cpu().numpy(), [32, 16], q, 0.125)
    close_attend(out, want, mag, BF)
