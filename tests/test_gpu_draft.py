"""A step of several tokens as it is used: a small model whose products have 4-bit weights reads two questions in one pass,
then answers with drafted trees -- reserve, append, attend in every layer, products, choice of a token after every node, the
path that is kept -- with some guesses right and some wrong.  What it answers has to be what the same model answers token by
token with attention of one new token per sequence, and the caches have to hold the same."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
L, HQ, HK, D, HIDDEN, VOCAB, PAGE, SEQS, WIDTH = 2, 8, 2, 64, 512, 997, 16, 2, 20
QUESTIONS = [37, 5]
NODES = 12


class Model:
    def __init__(self):
        from paper_2510_18269_b200 import oqm
        oqm.lib()
        self.oqm = oqm
        g = torch.Generator(device="cuda").manual_seed(1)

        def w4(n, k, group):
            unit = 1.5 / (4.6 * k ** 0.5)
            codes = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
            scale = (unit * (0.5 + torch.rand(n, k // group, generator=g, device="cuda"))).to(BF)
            return oqm.W4Matrix(codes, scale)                      # codes around 8
        self.emb = torch.randn(VOCAB, HIDDEN, generator=g, device="cuda").to(BF)
        self.qkv = [w4((HQ + 2 * HK) * D, HIDDEN, 128) for _ in range(L)]
        self.out = [w4(HIDDEN, HQ * D, 64) for _ in range(L)]
        self.up, self.down = [w4(4 * HIDDEN, HIDDEN, 32) for _ in range(L)], [w4(HIDDEN, 4 * HIDDEN, 128) for _ in range(L)]
        self.head = w4(VOCAB, HIDDEN, 128)
        self.bias = [torch.randn((HQ + 2 * HK) * D, generator=g, device="cuda").to(BF) for _ in range(L)]
        self.rope = oqm.Rope(oqm.stom_kv_frequencies(D, theta=1.0e4).cuda())

    def cache(self):
        c = type("Cache", (), {})()
        i32 = dict(dtype=torch.int32, device="cuda")
        c.k, c.v = (torch.zeros(L, SEQS * WIDTH + 3, PAGE, HK, D, dtype=BF, device="cuda") for _ in range(2))
        c.table, c.len = torch.full((SEQS, WIDTH), -1, **i32), torch.zeros(SEQS, **i32)
        c.refs, c.flags = torch.zeros(c.k.shape[1], **i32), torch.zeros(1, **i32)
        c.pool, c.seqs = self.oqm.KvPool(c.k, c.v), self.oqm.KvSeqs(c.table, c.len, c.refs)
        c.pages_ws = torch.empty(self.oqm.stom_kv_pages_workspace_bytes(c.pool, c.seqs), dtype=torch.uint8, device="cuda")
        rows = max(sum(QUESTIONS), SEQS * NODES)
        need = max(self.oqm.stom_kv_attend_tree_workspace_bytes(c.pool, c.seqs, rows, HQ),
                   self.oqm.stom_kv_attend_workspace_bytes(c.pool, c.seqs, HQ))
        c.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        return c

    def logits(self, c, token, pos, slot, seq, attend):
        """One pass over rows of tokens whose pages are there; attend(layer, q, out) is the attention."""
        o, n = self.oqm, token.shape[0]
        x = self.emb[token.long()]
        new = lambda *s: torch.empty(n, *s, dtype=BF, device="cuda")  # noqa: E731
        for l in range(L):
            qkv = new((HQ + 2 * HK) * D)
            o.stom_w4_linear(self.qkv[l], x, qkv, bias=self.bias[l], dev_flags=c.flags)
            qkv = qkv.view(n, HQ + 2 * HK, D)
            q, att = new(HQ, D), torch.zeros(n, HQ, D, dtype=BF, device="cuda")
            o.stom_kv_append(c.pool, c.seqs, l, self.rope, pos, slot, qkv[:, HQ:HQ + HK], qkv[:, HQ + HK:], q=qkv[:, :HQ], q_out=q,
                             seq=seq, dev_flags=c.flags)
            attend(l, q, att)
            h = new(HIDDEN)
            o.stom_w4_linear(self.out[l], att.view(n, -1), h, add=x, dev_flags=c.flags)
            up = new(4 * HIDDEN)
            o.stom_w4_linear(self.up[l], h, up, dev_flags=c.flags)
            o.stom_w4_linear(self.down[l], torch.nn.functional.silu(up), h, add=h, dev_flags=c.flags)   # onto itself
            x = h
        y = new(VOCAB)
        o.stom_w4_linear(self.head, x, y, dev_flags=c.flags)
        return y

    def greedy(self, y):
        token = torch.empty(y.shape[0], dtype=torch.int32, device="cuda")
        cold = torch.zeros(y.shape[0], device="cuda")
        self.oqm.stom_sample_tokens(y, None, token, temperature=cold)
        return token


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _read_questions(m, c):
    """The questions in one pass; the first token of each answer."""
    rng = np.random.default_rng(2)
    first = [0, QUESTIONS[0], sum(QUESTIONS)]
    m.oqm.stom_kv_reserve(c.pool, c.seqs, _ints(QUESTIONS), c.pages_ws, dev_flags=c.flags)
    pos = _ints([t for n in QUESTIONS for t in range(n)])
    seq = _ints([i for i, n in enumerate(QUESTIONS) for _ in range(n)])
    token = _ints(rng.integers(0, VOCAB, first[-1]))
    f = _ints(first)
    y = m.logits(c, token, pos, pos, seq, lambda l, q, out: m.oqm.stom_kv_attend_tree(
        c.pool, c.seqs, l, f, q, out, D ** -0.5, c.ws, dev_flags=c.flags))
    return m.greedy(y)[[QUESTIONS[0] - 1, first[-1] - 1]]


def _token_by_token(m, steps):
    c = m.cache()
    token = _read_questions(m, c)
    answers = [token.tolist()]
    for _ in range(steps):
        at = c.len.clone()
        m.oqm.stom_kv_reserve(c.pool, c.seqs, at + 1, c.pages_ws, dev_flags=c.flags)
        y = m.logits(c, token, at, at, None, lambda l, q, out: m.oqm.stom_kv_attend(
            c.pool, c.seqs, l, q, out, D ** -0.5, c.ws, dev_flags=c.flags))
        token = m.greedy(y)
        answers.append(token.tolist())
    torch.cuda.synchronize()
    assert c.flags.item() == 0
    return c, np.array(answers).T


def _rows(c, x, i, n):
    """The first n tokens of sequence i in all layers."""
    t = torch.arange(n, device="cuda")
    return x[:, c.table[i].long()[t // PAGE], t % PAGE].float()


@pytest.mark.parametrize("captured", [False, True])
def test_answers_with_drafts_are_those_without(captured):
    m = Model()
    steps = 40
    plain, answers = _token_by_token(m, steps)
    c = m.cache()
    pending = _read_questions(m, c)
    assert pending.tolist() == answers[:, 0].tolist()
    # what a pass works in: filled anew before every pass, so that a captured one can be replayed
    i32 = dict(dtype=torch.int32, device="cuda")
    first = _ints([0, NODES, 2 * NODES])
    parent, draft, seq = torch.zeros(2 * NODES, **i32), torch.zeros(2 * NODES, **i32), _ints([0] * NODES + [1] * NODES)
    depth = torch.zeros(2 * NODES, **i32)
    path, count, following = torch.zeros(2 * NODES, **i32), torch.zeros(2, **i32), torch.zeros(2, **i32)
    node = torch.arange(NODES, **i32).repeat(2)

    def step():
        base = c.len[seq.long()]
        m.oqm.stom_kv_reserve(c.pool, c.seqs, c.len + NODES, c.pages_ws, dev_flags=c.flags)
        y = m.logits(c, draft, base + depth, base + node, seq, lambda l, q, out: m.oqm.stom_kv_attend_tree(
            c.pool, c.seqs, l, first, q, out, D ** -0.5, c.ws, parent=parent, dev_flags=c.flags))
        m.oqm.stom_kv_accept(c.pool, c.seqs, first, draft, m.greedy(y), path, count, following, parent=parent, dev_flags=c.flags)

    rng = np.random.default_rng(3)
    done = [1, 1]                                                  # tokens known of each answer
    graph = None
    while min(done) < steps - 8:
        p, d, g = [], [], []
        for i in range(SEQS):
            # a tree whose path of `right` nodes holds what will be chosen; the others guess wrongly
            right = int(rng.integers(0, 6))
            par, dep, tok, good = [-1], [0], [answers[i, done[i] - 1]], [0]
            for j in range(1, NODES):
                grow = len(good) <= right and rng.random() < 0.6
                up = good[-1] if grow else int(rng.integers(0, j))
                par.append(up)
                dep.append(dep[up] + 1)
                true = answers[i, done[i] - 1 + dep[j]] if dep[j] + done[i] <= steps else 0
                tok.append(true if grow else (int(true) + 1 + j) % VOCAB)
                if grow:
                    good.append(j)
            p += par
            d += tok
            g += dep
        parent.copy_(_ints(p)), draft.copy_(_ints(d)), depth.copy_(_ints(g))
        before = c.len.clone()
        if captured and graph is not None:
            graph.replay()
        else:
            step()
        torch.cuda.synchronize()
        if captured and graph is None:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        assert c.flags.item() == 0
        for i in range(SEQS):
            n = int(count[i])
            way = path[i * NODES:i * NODES + n].tolist()
            kept = [d[i * NODES + j] for j in way]
            assert kept == answers[i, done[i] - 1:done[i] - 1 + n].tolist()
            assert int(following[i]) == answers[i, done[i] - 1 + n]
            # as far as the right guesses reached (a wrong one may be right by chance further down a wrong path: never kept)
            assert int(c.len[i]) == int(before[i]) + n
            done[i] += n
    held = {int(x) for row, n in zip(c.table.tolist(), c.len.tolist()) for x in row[:-(-n // PAGE)]}
    assert (c.refs > 0).sum().item() == len(held) and all(c.refs[x] == 1 for x in held)
    # the caches: the same tokens, computed in passes of other sizes; bf16 steps of values of about 1 to 4 through two layers
    for i in range(SEQS):
        n = min(int(c.len[i]), int(plain.len[i]))
        for a, b in ((c.k, plain.k), (c.v, plain.v)):
            x, y = _rows(c, a, i, n), _rows(plain, b, i, n)
            assert (x - y).abs().max() <= 2.0 ** -4 * max(1.0, y.abs().max().item()), (x - y).abs().max()
            assert (x[0] - y[0]).abs().max() <= 2.0 ** -7 * y[0].abs().max()          # the first layer: one rounding
