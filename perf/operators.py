"""Workloads of the answering side: rotary positions, the paged key-value cache and the choice of the next token.

After the memory has been searched, a language model answers over the reconstructed cache: the projections of new
tokens are (normalised and) rotated, keys and values go to pages, every new token attends over its pages, pages are
shared between candidate answers and moved together, and a token is drawn from the logits.  Each case below is one
such call at sizes a program meets; `run` makes it in plain torch operations or, with `own` set, through the library.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ESIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
DEV = "cuda"


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # the keys and queries of a whole reconstructed cache plus a question, one layer of the 7B shape
        dict(name="rotate-prompt", op="rotate", n=12583, hq=28, hk=4, d=128, rot=128, layout="half", norm=False,
             scaling="plain", far=13000, dtype="bf16"),
        # a short prompt of a model with per-head norms and a quarter of the head rotated in pairs, in binary32
        dict(name="rotate-norm-pairs", op="rotate", n=1771, hq=16, hk=8, d=64, rot=16, layout="pairs", norm=True,
             scaling="waves", far=900000, dtype="fp32"),
        # one decode step of one stream: the smallest call there is
        dict(name="append-one", op="append", n=1, seqs=1, page=50, hq=28, hk=4, d=128, rot=128, layout="half",
             norm=False, scaling="plain", far=13000, dtype="bf16"),
        # five prompts of unequal length in one call, 72B head counts, norms, pages of 16
        dict(name="append-prompts", op="append", n=4099, seqs=5, page=16, hq=64, hk=8, d=128, rot=128, layout="half",
             norm=True, scaling="linear", far=33000, dtype="fp16"),
        # one decode step over 251 retrieved groups and a question; a page is a frame's group of 50 tokens
        dict(name="attend-one-stream", op="attend", seqs=1, least=12583, most=12583, hq=28, hk=4, d=128, page=50,
             window=0, cap=0.0, dtype="bf16"),
        # a decode step of 64 streams of very unequal length, 72B head counts
        dict(name="attend-ragged", op="attend", seqs=64, least=17, most=16411, hq=64, hk=8, d=128, page=16,
             window=0, cap=0.0, dtype="bf16"),
        # many short conversations, some of them empty, odd page size
        dict(name="attend-short", op="attend", seqs=233, least=0, most=300, hq=16, hk=2, d=64, page=7,
             window=0, cap=0.0, dtype="fp16"),
        # sliding window and capped scores, wide heads
        dict(name="attend-window-cap", op="attend", seqs=19, least=1, most=9001, hq=8, hk=4, d=256, page=64,
             window=1000, cap=30.0, dtype="bf16"),
        # candidate answers: the last candidates are dropped, eight streams are forked eight times each, every
        # candidate gets room for its next token (a copy of the page it shares), all 28 layers
        dict(name="pages-branch", op="branch", parents=8, children=8, least=213, most=2950, page=50, layers=28, hk=4,
             d=128, dtype="bf16"),
        # half of the streams have ended and the pages of the others are moved together
        dict(name="pages-compact", op="compact", seqs=40, least=1, most=900, page=50, layers=28, hk=4, d=128,
             dtype="bf16"),
        # the next token of one stream
        dict(name="sample-one", op="sample", rows=1, n=128000, dtype="fp32", pick="usual", masked=False),
        # the next tokens of a batch with mixed settings, part of the vocabulary forbidden
        dict(name="sample-batch", op="sample", rows=128, n=151001, dtype="bf16", pick="mixed", masked=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend", "branch", "compact", "sample", "sample"])
    d = rng.choice([64, 128, 256])
    hk = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 4, 7, 8, 12])
    page = rng.choice([1, 7, 16, 32, 50, 64, 128])
    if op in ("rotate", "append"):
        c = dict(op=op, n=_log(rng, 1, 9000), hq=hk * g, hk=hk, d=d, rot=rng.choice([16, d // 2, d]),
                 layout=rng.choice(["half", "pairs"]), norm=rng.random() < 0.5,
                 scaling=rng.choice(["plain", "linear", "base", "waves"]), far=_log(rng, 100, 2000000))
        if d * hk * (g + 1) * c["n"] > 40 << 20:
            c["n"] = max(1, (40 << 20) // (d * hk * (g + 1)))
        if op == "rotate":
            c["dtype"] = rng.choice(["bf16", "fp16", "fp32"])
        else:
            c.update(seqs=min(c["n"], _log(rng, 1, 64)), page=page, dtype=rng.choice(["bf16", "fp16"]))
        return c
    if op == "attend":
        seqs = _log(rng, 1, 200)
        room = (1 << 30) // (seqs * hk * d * 4)                  # at most 1 GB of keys and values
        most = min(_log(rng, 1, 30000), max(1, room))
        return dict(op=op, seqs=seqs, least=rng.randint(0, most), most=most, hq=hk * g, hk=hk, d=d, page=page,
                    window=rng.choice([0, 0, _log(rng, 1, most)]), cap=rng.choice([0.0, 0.0, 20.0]),
                    dtype=rng.choice(["bf16", "fp16"]))
    if op in ("branch", "compact"):
        c = dict(op=op, least=rng.randint(1, 60), most=_log(rng, 61, 800), page=page, layers=_log(rng, 1, 28), hk=hk,
                 d=d, dtype=rng.choice(["bf16", "fp16"]))
        if op == "branch":
            c.update(parents=_log(rng, 1, 12), children=_log(rng, 1, 9))
        else:
            c.update(seqs=_log(rng, 2, 80))
        rows = c["parents"] * (1 + c["children"]) if op == "branch" else c["seqs"]
        c["layers"] = max(1, min(c["layers"], (1 << 30) // (rows * (c["most"] + page) * hk * d * 4)))
        return c
    return dict(op=op, rows=_log(rng, 1, 100), n=_log(rng, 2, 140000), dtype=rng.choice(["bf16", "fp16", "fp32"]),
                pick=rng.choice(["greedy", "plain", "top_k", "top_p", "min_p", "usual", "mixed"]),
                masked=rng.random() < 0.4)


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, shape, dt, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * scale).to(dt)


def _freq(c):
    """Angular step per position of every rotated pair (binary64), for the ways of reaching far positions."""
    r, theta, factor = c["rot"], 1.0e6, 8.0
    i = torch.arange(r // 2, dtype=torch.float64)
    if c["scaling"] == "base":
        theta *= factor ** (r / max(r - 2, 1))
    f = theta ** (-2.0 * i / r)
    if c["scaling"] == "linear":
        f = f / factor
    if c["scaling"] == "waves":
        turns = 8192.0 * f / (2.0 * math.pi)                     # turns over the length trained on
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    return f.to(DEV)


def _spread(lo, hi, n):
    """n lengths between lo and hi, many short and few long, the same for every seed."""
    return [lo + int(round((hi - lo) * ((i + 1.0) / n) ** 2)) if n > 1 else hi for i in range(n)]


def _pages_of(lens, page):
    return [(x + page - 1) // page for x in lens]


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _table(g, lens, page, spare):
    """A table of shuffled pages for these lengths: (table, refs)."""
    held = _pages_of(lens, page)
    total = sum(held)
    order = torch.randperm(total + spare, generator=g, device=DEV)[:total].to(torch.int32)
    width = max(1, max(held))
    cols = torch.arange(width, device=DEV)[None, :]
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    table[cols < _ints(held)[:, None]] = order
    refs = torch.zeros(total + spare, dtype=torch.int32, device=DEV)
    refs[order.long()] = 1
    return table, refs


def _shuffled(g, v):
    p = torch.randperm(len(v), generator=g, device=DEV).tolist()
    return [v[i] for i in p]


def prepare(case, seed):
    c, g = case, _gen(seed)
    dt = DT[c["dtype"]]
    s = dict(case=c)
    if c["op"] in ("rotate", "append"):
        n = c["n"]
        s["q"], s["k"] = _randn(g, (n, c["hq"], c["d"]), dt), _randn(g, (n, c["hk"], c["d"]), dt)
        s["q_out"] = torch.empty_like(s["q"])
        s["freq"] = _freq(c)
        s["qw"] = 1.0 + 0.2 * torch.randn(c["d"], generator=g, device=DEV) if c["norm"] else None
        s["kw"] = 1.0 + 0.2 * torch.randn(c["d"], generator=g, device=DEV) if c["norm"] else None
        s["mag"] = 1.0
        if c["op"] == "rotate":
            s["k_out"] = torch.empty_like(s["k"])
            first = int(torch.randint(0, max(1, c["far"] - n), (1,), generator=g, device=DEV))
            s["pos"] = torch.arange(first, first + n, dtype=torch.int32, device=DEV)
            return s
        s["v"] = _randn(g, (n, c["hk"], c["d"]), dt)
        # the new tokens of a sequence stand behind what it holds already
        b = c["seqs"]
        count = [n // b + (1 if i < n % b else 0) for i in range(b)]
        if b > 1:
            for i in range(0, b - 1, 2):                         # unequal prompts
                m = count[i] // 2
                count[i], count[i + 1] = count[i] - m, count[i + 1] + m
        had = torch.randint(0, 400, (b,), generator=g, device=DEV).tolist()
        lens = [x + y for x, y in zip(had, count)]
        s["table"], refs = _table(g, [399 + max(count)] * b, c["page"], 3)
        s["len"] = _ints(lens)
        shape = (1, refs.numel(), c["page"], c["hk"], c["d"])
        s["pool_k"], s["pool_v"] = _randn(g, shape, dt), _randn(g, shape, dt)
        s["seq"] = torch.repeat_interleave(torch.arange(b, device=DEV), _ints(count)).to(torch.int32)
        starts = torch.cumsum(_ints(count), 0) - _ints(count)
        at = torch.arange(n, device=DEV) - starts[s["seq"].long()]
        s["slot"] = (at + _ints(had)[s["seq"].long()]).to(torch.int32)
        s["pos"] = (s["slot"] + max(0, c["far"] - 500 - max(count))).to(torch.int32)
        return s
    if c["op"] == "attend":
        lens = _shuffled(g, _spread(c["least"], c["most"], c["seqs"]))
        s["table"], refs = _table(g, lens, c["page"], 5)
        s["len"] = _ints(lens)
        shape = (1, refs.numel(), c["page"], c["hk"], c["d"])
        s["pool_k"], s["pool_v"] = _randn(g, shape, dt), _randn(g, shape, dt)
        s["q"] = _randn(g, (c["seqs"], c["hq"], c["d"]), dt, 1.5)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(c["seqs"], c["hq"], dtype=torch.float32, device=DEV)
        s["scale"] = 1.0 / math.sqrt(c["d"])
        return s
    if c["op"] == "branch":
        r, f = c["parents"], c["children"]
        lens = _shuffled(g, _spread(c["least"], c["most"], r))
        spare = r * f * 2 + 3
        table, refs = _table(g, lens, c["page"], spare)
        b = r * (1 + f)
        width = table.shape[1] + 1
        s["table"] = torch.full((b, width), -1, dtype=torch.int32, device=DEV)
        s["table"][:r, :-1] = table
        s["refs"] = refs
        s["len"] = _ints(lens + [0] * (r * f))
        s["parent"] = _ints([-1] * r + [i % r for i in range(r * f)])
        s["drop"] = _ints([0] * r + [1] * (r * f))
        s["want"] = _ints([0] * r + [lens[i % r] + 1 for i in range(r * f)])
    elif c["op"] == "compact":
        lens = _shuffled(g, _spread(c["least"], c["most"], c["seqs"]))
        alive = [1 if i % 2 else 0 for i in range(c["seqs"])]
        alive = _shuffled(g, alive)
        table, refs = _table(g, lens, c["page"], 9)
        gone = _ints(alive) == 0
        held = _ints(_pages_of(lens, c["page"]))
        dead = table[gone[:, None] & (torch.arange(table.shape[1], device=DEV)[None] < held[:, None])]
        refs[dead.long()] = 0
        table[gone] = -1
        s["table"], s["refs"], s["len"] = table, refs, _ints(lens) * _ints(alive)
        s["table_out"], s["refs_out"] = torch.empty_like(table), torch.empty_like(refs)
        s["live"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    else:
        rows, n = c["rows"], c["n"]
        x = torch.randn(rows, n, generator=g, device=DEV) * 2.5
        peak = torch.randint(0, n, (rows, 12), generator=g, device=DEV)
        x.scatter_add_(1, peak, torch.rand(rows, 12, generator=g, device=DEV) * 12.0)
        if c["masked"]:
            x[:, torch.rand(n, generator=g, device=DEV) < 0.3] = -math.inf
            x[:, n // 2] = 1.0                                   # something is always allowed
        s["x"] = x.to(dt)
        del x
        one = torch.ones(rows, device=DEV)
        which = torch.randint(0, 6, (rows,), generator=g, device=DEV)
        has = {p: torch.zeros(rows, dtype=torch.bool, device=DEV) for p in ("greedy", "top_k", "top_p", "min_p")}
        if c["pick"] == "mixed":
            has = dict(greedy=which == 0, top_k=(which == 1) | (which == 4), top_p=(which == 2) | (which == 4),
                       min_p=which == 3)
        elif c["pick"] == "usual":
            has["top_k"], has["top_p"] = ~has["top_k"], ~has["top_p"]
        elif c["pick"] != "plain":
            has[c["pick"]] = ~has[c["pick"]]
        warm = 0.5 + torch.rand(rows, generator=g, device=DEV)
        s["temperature"] = torch.where(has["greedy"], 0.0 * one, warm)
        s["top_k"] = torch.where(has["top_k"], torch.randint(1, 120, (rows,), generator=g, device=DEV), 0).to(torch.int32)
        s["top_p"] = torch.where(has["top_p"], 0.3 + 0.69 * torch.rand(rows, generator=g, device=DEV), one)
        s["min_p"] = torch.where(has["min_p"], 0.2 * torch.rand(rows, generator=g, device=DEV), 0.0 * one)
        s["u"] = torch.rand(rows, generator=g, device=DEV)
        s["token"] = torch.empty(rows, dtype=torch.int32, device=DEV)
        s["kept"] = torch.empty(rows, dtype=torch.int32, device=DEV)
        s["logprob"] = torch.empty(rows, dtype=torch.float32, device=DEV)
        return s
    shape = (c["layers"], s["refs"].numel(), c["page"], c["hk"], c["d"])
    s["pool_k"], s["pool_v"] = _randn(g, shape, dt), _randn(g, shape, dt)
    return s


# ---------------------------------------------------------------- plain forms

def _turn(x, pos, freq, layout, weight, mag, eps=1e-6):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + eps) * weight
    angle = pos.double()[:, None] * freq[None, :]
    cos, sin = (angle.cos() * mag).float()[:, None, :], (angle.sin() * mag).float()[:, None, :]
    h = freq.numel()
    a, b = (y[..., :h], y[..., h:2 * h]) if layout == "half" else (y[..., 0:2 * h:2], y[..., 1:2 * h:2])
    p, q = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([p, q], -1) if layout == "half" else torch.stack([p, q], -1).flatten(-2)
    return torch.cat([turned, y[..., 2 * h:]], -1).to(x.dtype)


def _attend(s):
    c, q, table = s["case"], s["q"], s["table"].long().clamp(min=0)
    b, hk, d = c["seqs"], c["hk"], c["d"]
    k = s["pool_k"][0][table].reshape(b, -1, hk, d).permute(0, 2, 3, 1).float()
    x = torch.matmul(q.float().view(b, hk, -1, d), k) * s["scale"]
    del k
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    t = torch.arange(x.shape[-1], device=DEV)[None, :]
    n = s["len"].long()[:, None]
    seen = t < n
    if c["window"]:
        seen = seen & (t >= n - c["window"])
    x = torch.where(seen[:, None, None, :], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    z = w.sum(-1, keepdim=True)
    v = s["pool_v"][0][table].reshape(b, -1, hk, d).permute(0, 2, 1, 3).float()
    o = torch.matmul(w, v) / torch.where(z == 0, 1.0, z)
    s["out"].copy_(o.view(b, c["hq"], d))
    s["lse"].copy_((top + torch.log(z)).view(b, c["hq"]))


def _held(n, page):
    return (n + page - 1) // page


def _branch(s):
    c, table, refs, n = s["case"], s["table"], s["refs"], s["len"]
    page, cols = c["page"], torch.arange(s["table"].shape[1], device=DEV)[None, :]
    # free
    gone = s["drop"] != 0
    mine = table[gone[:, None] & (cols < _held(n, page)[:, None])].long()
    refs.scatter_add_(0, mine, torch.full_like(mine, -1, dtype=torch.int32))
    table.masked_fill_(gone[:, None], -1)
    n.masked_fill_(gone, 0)
    # fork
    made = (s["parent"] >= 0) & (n == 0)
    of = s["parent"].clamp(min=0).long()
    copied = torch.where(cols < _held(n[of], page)[:, None], table[of], -1)
    table.copy_(torch.where(made[:, None], copied, table))
    mine = copied[made[:, None] & (copied >= 0)].long()
    refs.scatter_add_(0, mine, torch.ones_like(mine, dtype=torch.int32))
    n.copy_(torch.where(made, n[of], n))
    # reserve: pages for the new length; a partly filled page that others hold too is copied first, but the last of
    # the growing rows keeps it where no row stays behind
    grow = s["want"] > n
    held = _held(n, page)
    last = table.gather(1, (held - 1).clamp(min=0).long()[:, None])[:, 0]
    part = grow & (n % page != 0)
    share = torch.where(part, last, -1)
    same = (share[:, None] == share[None, :]) & part[:, None] & part[None, :]
    later = torch.triu(same, 1).any(1)
    holders = refs[last.clamp(min=0).long()]
    copies = part & (holders > 1) & (later | (holders > same.sum(1)))
    need = torch.where(grow, _held(s["want"], page) - held + copies.int(), 0)
    first = torch.cumsum(need, 0) - need
    free = torch.nonzero(refs == 0)[:, 0].to(torch.int32)
    begin = held - copies.int()                                  # first column that gets a new page
    takes = grow[:, None] & (cols >= begin[:, None]) & (cols < _held(s["want"], page)[:, None])
    at = (first[:, None] + cols - begin[:, None]).long()
    fresh = free[at.clamp(0, free.numel() - 1)]
    src, dst, used = last[copies].long(), fresh.gather(1, begin.clamp(min=0).long()[:, None])[:, 0][copies].long(), (n % page)[copies]
    refs.scatter_add_(0, src, torch.full_like(src, -1, dtype=torch.int32))
    refs[fresh[takes].long()] = 1
    table.copy_(torch.where(takes, fresh, table))
    tok = torch.arange(page, device=DEV)
    i, j = torch.nonzero(tok[None, :] < used[:, None], as_tuple=True)
    s["pool_k"][:, dst[i], j] = s["pool_k"][:, src[i], j]
    s["pool_v"][:, dst[i], j] = s["pool_v"][:, src[i], j]
    n.copy_(torch.where(grow, s["want"], n))


def _compact(s):
    c, refs = s["case"], s["refs"]
    live = refs > 0
    count = live.sum()
    here = torch.arange(refs.numel(), device=DEV)
    src, dst = here[live & (here >= count)], here[~live & (here < count)]
    to = here.clone()
    to[src] = dst
    cols = torch.arange(s["table"].shape[1], device=DEV)[None, :]
    moved = to[s["table"].clamp(min=0).long()].to(torch.int32)
    s["table_out"].copy_(torch.where(cols < _held(s["len"], c["page"])[:, None], moved, -1))
    s["refs_out"].zero_()
    s["refs_out"][to[live]] = refs[live]
    s["live"].copy_(count)
    s["pool_k"][:, dst] = s["pool_k"][:, src]
    s["pool_v"][:, dst] = s["pool_v"][:, src]


def _sample(s):
    # in 64 bits: a draw may fall next to a border between two tokens
    x = s["x"].double()
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    top, t = x[:, :1], s["temperature"].double()[:, None]
    cold = t <= 0
    w = torch.where(x == -math.inf, 0.0, torch.exp((x - top) / torch.where(cold, 1.0, t)))
    rank = torch.arange(x.shape[1], device=DEV)[None, :]
    k = s["top_k"].long()[:, None]
    w = torch.where(cold & (rank > 0) | (k > 0) & (rank >= k), 0.0, w)
    upto = torch.cumsum(w, 1)
    before = torch.cat([torch.zeros_like(upto[:, :1]), upto[:, :-1]], 1)
    p = s["top_p"].double()[:, None]
    keep = (w > 0) & ((p >= 1) | (before < p * upto[:, -1:])) & (w >= s["min_p"].double()[:, None]) | (rank == 0)
    count = keep.sum(1)
    mass = upto.gather(1, count[:, None] - 1)
    aim = s["u"].double()[:, None] * mass
    j = torch.minimum((upto <= aim).sum(1), count - 1)[:, None]
    s["token"].copy_(order.gather(1, j)[:, 0])
    s["kept"].copy_(count)
    s["logprob"].copy_((torch.log(w.gather(1, j)) - torch.log(mass))[:, 0])


# ---------------------------------------------------------------- one pass

def _own(s):
    from paper_2510_18269_b200 import oqm
    c = s["case"]
    # the descriptors and the workspace are made once by a program and kept beside its cache
    if c["op"] in ("rotate", "append") and "rope" not in s:
        s["rope"] = oqm.Rope(s["freq"], layout=oqm.ROPE_HALF if c["layout"] == "half" else oqm.ROPE_PAIRS,
                             magnitude=s["mag"])
    if "pool_k" in s and "pool" not in s:
        s["pool"] = oqm.KvPool(s["pool_k"], s["pool_v"])
        s["seqs"] = oqm.KvSeqs(s["table"], s["len"], s.get("refs"))
        need = (oqm.stom_kv_attend_workspace_bytes(s["pool"], s["seqs"], c["hq"]) if c["op"] == "attend" else
                oqm.stom_kv_pages_workspace_bytes(s["pool"], s["seqs"]))
        s["ws"] = torch.zeros(need, dtype=torch.uint8, device=DEV)
    if c["op"] == "sample":
        oqm.stom_sample_tokens(s["x"], s["u"], s["token"], temperature=s["temperature"], top_k=s["top_k"],
                               top_p=s["top_p"], min_p=s["min_p"], logprob=s["logprob"], kept=s["kept"])
        return
    if c["op"] == "rotate":
        oqm.stom_kv_rotate(s["rope"], s["pos"], q=s["q"], q_out=s["q_out"], k=s["k"], k_out=s["k_out"],
                           q_weight=s["qw"], k_weight=s["kw"], eps=1e-6)
        return
    pool, seqs = s["pool"], s["seqs"]
    if c["op"] == "append":
        oqm.stom_kv_append(pool, seqs, 0, s["rope"], s["pos"], s["slot"], s["k"], s["v"], q=s["q"], q_out=s["q_out"],
                           seq=s["seq"], q_weight=s["qw"], k_weight=s["kw"], eps=1e-6)
    elif c["op"] == "attend":
        oqm.stom_kv_attend(pool, seqs, 0, s["q"], s["out"], s["scale"], s["ws"], lse=s["lse"], softcap=c["cap"],
                           window=c["window"])
    elif c["op"] == "branch":
        oqm.stom_kv_free(pool, seqs, s["drop"])
        oqm.stom_kv_fork(pool, seqs, s["parent"])
        oqm.stom_kv_reserve(pool, seqs, s["want"], s["ws"])
    else:
        oqm.stom_kv_compact(pool, seqs, s["table_out"], s["refs_out"], s["live"], s["ws"])


def _plain(s):
    c = s["case"]
    if c["op"] == "sample":
        _sample(s)
    elif c["op"] == "attend":
        _attend(s)
    elif c["op"] == "branch":
        _branch(s)
    elif c["op"] == "compact":
        _compact(s)
    else:
        s["q_out"].copy_(_turn(s["q"], s["pos"], s["freq"], c["layout"], s["qw"], s["mag"]))
        k = _turn(s["k"], s["pos"], s["freq"], c["layout"], s["kw"], s["mag"])
        if c["op"] == "rotate":
            s["k_out"].copy_(k)
        else:
            slot = s["slot"].long()
            page = s["table"][s["seq"].long(), slot // c["page"]].long()
            s["pool_k"][0, page, slot % c["page"]] = k
            s["pool_v"][0, page, slot % c["page"]] = s["v"]


OUTPUTS = {
    "rotate": ("q_out", "k_out"), "append": ("q_out", "pool_k", "pool_v"), "attend": ("out", "lse"),
    "branch": ("table", "len", "refs", "pool_k", "pool_v"),
    "compact": ("table_out", "refs_out", "live", "pool_k", "pool_v"), "sample": ("token", "kept", "logprob"),
}


def run(state):
    if own:
        _own(state)
    else:
        _plain(state)
    return [state[k] for k in OUTPUTS[state["case"]["op"]]]


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "sample":
        return dict(bytes=c["rows"] * (c["n"] * ESIZE[c["dtype"]] + 32), flops=0)
    row = c["hk"] * c["d"] * ESIZE[c["dtype"]]
    if c["op"] in ("rotate", "append"):
        moved = 2 * c["n"] * (c["hq"] * c["d"] * ESIZE[c["dtype"]] + row * (1 if c["op"] == "rotate" else 2))
        return dict(bytes=moved + 4 * c["n"], flops=c["n"] * (c["hq"] + c["hk"]) * (3 * c["rot"] + (4 * c["d"] if c["norm"] else 0)))
    if c["op"] == "attend":
        lens = _spread(c["least"], c["most"], c["seqs"])
        seen = sum(min(x, c["window"]) if c["window"] else x for x in lens)
        ends = c["seqs"] * c["hq"] * (2 * c["d"] * ESIZE[c["dtype"]] + 4)
        return dict(bytes=2 * seen * row + ends, flops=4 * seen * c["hq"] * c["d"])
    if c["op"] == "branch":
        lens = _spread(c["least"], c["most"], c["parents"])
        used = sum(x % c["page"] for x in lens) * c["children"]
        ints = c["parents"] * (1 + c["children"]) * 8 + sum(_pages_of(lens, c["page"])) * 4 * (1 + 2 * c["children"])
        return dict(bytes=c["layers"] * 2 * 2 * used * row + ints, flops=0)
    held = sum(_pages_of(_spread(c["least"], c["most"], c["seqs"]), c["page"]))
    moved = held // 4                                            # half of the pages live, half of those stand behind
    return dict(bytes=c["layers"] * 2 * 2 * moved * c["page"] * row + 16 * held, flops=0)


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _exact_turn(x, pos, freq, layout, weight, mag):
    z = x.double()
    if weight is not None:
        z = z / torch.sqrt((z * z).sum(-1, keepdim=True) / z.shape[-1] + 1e-6) * weight.double()
    h = freq.numel()
    turn = torch.polar(torch.full((pos.numel(), 1, h), float(mag), dtype=torch.float64, device=DEV),
                       (pos.double()[:, None] * freq)[:, None, :])
    if layout == "half":
        c = torch.complex(z[..., :h].contiguous(), z[..., h:2 * h].contiguous()) * turn
        z[..., :h], z[..., h:2 * h] = c.real, c.imag
    else:
        c = torch.view_as_complex(z[..., :2 * h].reshape(*z.shape[:-1], h, 2).contiguous()) * turn
        z[..., :2 * h] = torch.view_as_real(c).flatten(-2)
    return z


def _exact_attend(s):
    c = s["case"]
    out = torch.zeros(c["seqs"], c["hq"], c["d"], dtype=torch.float64, device=DEV)
    lse = torch.full((c["seqs"], c["hq"]), -math.inf, dtype=torch.float64, device=DEV)
    g = c["hq"] // c["hk"]
    for i, n in enumerate(s["len"].tolist()):
        first = max(0, n - c["window"]) if c["window"] else 0
        if n <= first:
            continue
        t = torch.arange(first, n, device=DEV)
        page = s["table"][i].long()[t // c["page"]]
        k, v = s["pool_k"][0, page, t % c["page"]].double(), s["pool_v"][0, page, t % c["page"]].double()
        for h in range(c["hk"]):
            x = s["q"][i, h * g:(h + 1) * g].double() @ k[:, h].T * s["scale"]
            if c["cap"]:
                x = torch.tanh(x / c["cap"]) * c["cap"]
            lse[i, h * g:(h + 1) * g] = torch.logsumexp(x, 1)
            out[i, h * g:(h + 1) * g] = torch.softmax(x, 1) @ v[:, h]
    return [out, lse]


def _exact_branch(s):
    c = s["case"]
    page = c["page"]
    table, n, refs = s["table"].tolist(), s["len"].tolist(), s["refs"].tolist()
    parent, drop, want = s["parent"].tolist(), s["drop"].tolist(), s["want"].tolist()
    for i in range(len(n)):
        if drop[i]:
            for j in range(-(-n[i] // page)):
                refs[table[i][j]] -= 1
            table[i], n[i] = [-1] * len(table[i]), 0
    before = list(n)
    for i in range(len(n)):
        if parent[i] >= 0 and before[i] == 0:
            m = -(-before[parent[i]] // page)
            table[i], n[i] = table[parent[i]][:m] + [-1] * (len(table[i]) - m), before[parent[i]]
            for j in range(m):
                refs[table[i][j]] += 1
    free = [p for p, r in enumerate(refs) if r == 0]
    for i in range(len(n)):
        if want[i] <= n[i]:
            continue
        m = -(-n[i] // page)
        if n[i] % page and refs[table[i][m - 1]] > 1:
            old, new = table[i][m - 1], free.pop(0)
            refs[old], refs[new], table[i][m - 1] = refs[old] - 1, 1, new
            for pool in (s["pool_k"], s["pool_v"]):
                pool[:, new, :n[i] % page] = pool[:, old, :n[i] % page]
        for j in range(m, -(-want[i] // page)):
            table[i][j] = free.pop(0)
            refs[table[i][j]] = 1
        n[i] = want[i]
    return [_ints(table), _ints(n), _ints(refs), s["pool_k"], s["pool_v"]]


def _exact_compact(s):
    table, refs, n = s["table"].tolist(), s["refs"].tolist(), s["len"].tolist()
    live = sum(r > 0 for r in refs)
    hole, to = 0, {}
    out = [0] * len(refs)
    for p, r in enumerate(refs):
        if r > 0:
            to[p] = p
            if p >= live:
                while refs[hole] > 0:
                    hole += 1
                to[p], hole = hole, hole + 1
                for pool in (s["pool_k"], s["pool_v"]):
                    pool[:, to[p]] = pool[:, p]
            out[to[p]] = r
    moved = [[to[p] if j < -(-n[i] // s["case"]["page"]) else -1 for j, p in enumerate(row)] for i, row in enumerate(table)]
    return [_ints(moved), _ints(out), _ints([live]), s["pool_k"], s["pool_v"]]


def _exact_sample(s):
    import numpy as np
    x = s["x"].double().cpu().numpy()
    par = [s[k].double().cpu().numpy() for k in ("temperature", "top_k", "top_p", "min_p", "u")]
    token, kept, logprob = [], [], []
    for i in range(x.shape[0]):
        t, k, p, m, u = (float(v[i]) for v in par)
        order = np.argsort(-x[i], kind="stable")
        order = order[x[i][order] > -math.inf]
        if t <= 0:
            order = order[:1]
        elif k > 0:
            order = order[:int(k)]
        w = np.exp((x[i][order] - x[i][order[0]]) / (t if t > 0 else 1.0))
        order, w = order[w > 0], w[w > 0]
        sums = np.cumsum(w)
        count = len(w)
        if p < 1:
            count = min(count, int(np.searchsorted(sums, p * sums[-1], side="left")) + 1)
        count = max(1, min(count, int((w >= m).sum())))
        j = min(int(np.searchsorted(sums[:count], u * sums[count - 1], side="right")), count - 1)
        token.append(int(order[j]))
        kept.append(count)
        logprob.append(math.log(w[j] / sums[count - 1]))
    return [_ints(token), _ints(kept), torch.tensor(logprob, dtype=torch.float64, device=DEV)]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("rotate", "append"):
        q = _exact_turn(s["q"], s["pos"], s["freq"], case["layout"], s["qw"], s["mag"])
        k = _exact_turn(s["k"], s["pos"], s["freq"], case["layout"], s["kw"], s["mag"])
        if case["op"] == "rotate":
            return [q, k]
        pool_k, pool_v = s["pool_k"].double(), s["pool_v"].double()
        slot = s["slot"].long()
        page = s["table"][s["seq"].long(), slot // case["page"]].long()
        pool_k[0].index_put_((page, slot % case["page"]), k)
        pool_v[0].index_put_((page, slot % case["page"]), s["v"].double())
        return [q, pool_k, pool_v]
    return {"attend": _exact_attend, "branch": _exact_branch, "compact": _exact_compact,
            "sample": _exact_sample}[case["op"]](s)
