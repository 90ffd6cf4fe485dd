"""Workloads of a step that takes several tokens of a sequence at once: attention of a tree of drafted tokens (or of a
question's tokens) over the paged cache, the acceptance of a drafted path, and products with 4-bit weights.

A model that answers over the reconstructed cache may be given several tokens to look at in one pass: the question
itself, or guesses of the next tokens, of which the pass keeps those that it would have chosen.  The weights of such a
pass are read once for all its tokens.  Each case below is one such call at sizes a program meets; `run` makes it in plain
torch operations or, with `own` set, through the library.
"""
import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ESIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
DEV = "cuda"


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # five tokens guessed ahead of one stream over a whole reconstructed cache, one after another: the smallest
        # verification there is
        dict(name="tree-chain-one", op="tree", seqs=1, least=12583, most=12583, nodes_least=5, nodes_most=5, shape="path",
             hq=28, hk=4, d=128, page=50, window=0, cap=0.0, dtype="bf16"),
        # a tree of 64 guesses over the same cache
        dict(name="tree-one-stream", op="tree", seqs=1, least=12583, most=12583, nodes_least=64, nodes_most=64, shape="tree",
             hq=28, hk=4, d=128, page=50, window=0, cap=0.0, dtype="bf16"),
        # a server's batch of unequal streams with unequal trees, 72B head counts, pages of 16
        dict(name="tree-batch", op="tree", seqs=48, least=17, most=8011, nodes_least=1, nodes_most=33, shape="tree",
             hq=64, hk=8, d=128, page=16, window=0, cap=0.0, dtype="fp16"),
        # a model with wide heads, a window and capped scores
        dict(name="tree-window-cap", op="tree", seqs=13, least=0, most=5003, nodes_least=3, nodes_most=41, shape="tree",
             hq=8, hk=4, d=256, page=64, window=1000, cap=30.0, dtype="bf16"),
        # questions read over retrieved caches: many new tokens each, causal
        dict(name="prefill-questions", op="tree", seqs=3, least=3200, most=12544, nodes_least=201, nodes_most=1201,
             shape="chain", hq=28, hk=4, d=128, page=50, window=0, cap=0.0, dtype="bf16"),
        # the accepted path of one stream's tree, all layers of the 7B shape
        dict(name="accept-one", op="accept", seqs=1, least=701, most=701, nodes=64, depth=6, page=50, layers=28, hk=4, d=128,
             dtype="bf16"),
        # a batch of them
        dict(name="accept-batch", op="accept", seqs=40, least=5, most=390, nodes=33, depth=5, page=16, layers=28, hk=4, d=128,
             dtype="bf16"),
        # one token's queries, keys and values: 28 + 4 + 4 heads from a hidden width of 28 heads
        dict(name="w4-one-qkv", op="w4", rows=1, n=4608, k=3584, group=128, zero=True, bias=True, add=False, meta="bf16",
             dtype="bf16"),
        # one token's widest product
        dict(name="w4-one-wide", op="w4", rows=1, n=28672, k=3584, group=64, zero=True, bias=False, add=False, meta="fp16",
             dtype="fp16"),
        # a drafted tree on the way back from the widest layer, onto the residual stream
        dict(name="w4-tree-down", op="w4", rows=64, n=3584, k=14336, group=128, zero=True, bias=False, add=True, meta="bf16",
             dtype="bf16"),
        # few tokens, codes around 8 without offsets, small groups, an odd number of outputs, the 72B width
        dict(name="w4-few-odd", op="w4", rows=13, n=10007, k=8192, group=32, zero=False, bias=True, add=True, meta="fp32",
             dtype="fp16"),
        # the logits of a drafted chain over an odd vocabulary: the largest weights
        dict(name="w4-logits", op="w4", rows=5, n=151001, k=3584, group=128, zero=True, bias=False, add=False, meta="bf16",
             dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "accept", "w4", "w4", "w4"])
    if op == "tree":
        d, hk, g = rng.choice([64, 128, 256]), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 7, 8, 12])
        shape = rng.choice(["path", "tree", "tree", "chain"])
        seqs = _log(rng, 1, 6 if shape == "chain" else 80)
        nodes = _log(rng, 1, 1500 if shape == "chain" else 160)
        room = (400 << 20) // (seqs * hk * d * 4)                # at most 400 MB of keys and values
        most = min(_log(rng, 1, 20000), max(1, room))
        # at most 10^11 multiply-adds
        nodes = max(1, min(nodes, 10 ** 11 // (2 * d * hk * g * seqs * (most + nodes))))
        return dict(op=op, seqs=seqs, least=rng.randint(0, most), most=most, nodes_least=rng.randint(1, nodes),
                    nodes_most=nodes, shape=shape, hq=hk * g, hk=hk, d=d, page=rng.choice([1, 7, 16, 32, 50, 64, 128]),
                    window=rng.choice([0, 0, _log(rng, 1, most + nodes)]), cap=rng.choice([0.0, 0.0, 20.0]),
                    dtype=rng.choice(["bf16", "fp16"]))
    if op == "accept":
        depth = rng.randint(1, 8)
        c = dict(op=op, seqs=_log(rng, 1, 60), least=rng.randint(0, 60), most=_log(rng, 61, 800),
                 nodes=rng.randint(2 * depth + 1, 100), depth=depth, page=rng.choice([1, 7, 16, 32, 50, 64, 128]),
                 layers=_log(rng, 1, 40), hk=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128, 256]),
                 dtype=rng.choice(["bf16", "fp16"]))
        per = c["seqs"] * (c["most"] + c["nodes"] + c["page"]) * c["hk"] * c["d"] * 4
        c["layers"] = max(1, min(c["layers"], (1 << 30) // per))
        return c
    group = rng.choice([32, 64, 128])
    rows, n, k = _log(rng, 1, 200), _log(rng, 1, 150000), group * _log(rng, 1, 16000 // group)
    n = max(1, min(n, 5 * 10 ** 8 // k, 2 * 10 ** 10 // (rows * k)))
    return dict(op=op, rows=rows, n=n, k=k, group=group, zero=rng.random() < 0.6, bias=rng.random() < 0.4,
                add=rng.random() < 0.4, meta=rng.choice(["bf16", "fp16", "fp32"]), dtype=rng.choice(["bf16", "fp16"]))


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, shape, dt, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * scale).to(dt)


def _spread(lo, hi, n):
    """n lengths between lo and hi, many short and few long, the same for every seed."""
    return [lo + int(round((hi - lo) * ((i + 1.0) / n) ** 2)) if n > 1 else hi for i in range(n)]


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _held(n, page):
    return -(-n // page)


def _tree(rng, n, shape):
    """Parents of n nodes: a path, or a tree in which most nodes hang from one of the last few."""
    if shape != "tree":
        return list(range(-1, n - 1))
    return [-1] + [max(0, j - 1 - min(int(rng.expovariate(0.15)), j - 1)) for j in range(1, n)]


def _lens(c, seed):
    """Lengths with the new tokens, and how many of them are new."""
    rng = random.Random(seed)
    had = _spread(c["least"], c["most"], c["seqs"])
    new = _spread(c["nodes_least"], c["nodes_most"], c["seqs"])
    rng.shuffle(had)
    rng.shuffle(new)
    return [a + b for a, b in zip(had, new)], new, rng


def _prepare_tree(c, seed, g, dt):
    lens, new, rng = _lens(c, seed)
    held = [_held(x, c["page"]) for x in lens]
    total = sum(held) + 5
    order = torch.randperm(total, generator=g, device=DEV)[:sum(held)].to(torch.int32)
    width = max(held)
    table = torch.full((c["seqs"], width), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(width, device=DEV)[None, :] < _ints(held)[:, None]] = order
    n = sum(new)
    first = [sum(new[:i]) for i in range(c["seqs"] + 1)]
    parent = None if c["shape"] == "chain" else _ints([p for m in new for p in _tree(rng, m, c["shape"])])
    s = dict(case=c, lens=lens, first_host=first, table=table, len=_ints(lens), first=_ints(first), parent=parent)
    shape = (1, total, c["page"], c["hk"], c["d"])
    s["pool_k"], s["pool_v"] = _randn(g, shape, dt), _randn(g, shape, dt)
    s["q"] = _randn(g, (n, c["hq"], c["d"]), dt, 1.5)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(n, c["hq"], dtype=torch.float32, device=DEV)
    s["scale"] = 1.0 / math.sqrt(c["d"])
    return s


def _prepare_accept(c, seed, g, dt):
    rng = random.Random(seed)
    b, n, page = c["seqs"], c["nodes"], c["page"]
    had = _spread(c["least"], c["most"], b)
    rng.shuffle(had)
    lens = [x + n for x in had]
    # pages of a context are anywhere; those that only drafted tokens use are taken in order
    firm, all_ = [_held(x + 1, page) for x in had], [_held(x, page) for x in lens]
    loose = sum(all_) - sum(firm)
    total = sum(all_) + 5
    ids = list(range(total))
    draft_ids, rest = ids[:loose], ids[loose:]
    rng.shuffle(rest)
    width = max(all_)
    rows = []
    for i in range(b):
        rows.append([rest.pop() for _ in range(firm[i])] + [draft_ids.pop(0) for _ in range(all_[i] - firm[i])])
    for p in rest:                                               # other streams hold the rest
        assert p >= loose
    refs = [1] * total
    table = [r + [-1] * (width - len(r)) for r in rows]
    # trees whose first guesses fail and whose later ones hold for one to `depth` steps
    parents, draft, chosen = [], [], []
    for i in range(b):
        p = [-1] + [0] * c["depth"]
        while len(p) < n:
            j = len(p)
            p.append(rng.choice([0] + list(range(c["depth"] + 1, j))) if j > c["depth"] + 1 else 0)
        tok = [rng.randint(0, 150000) for _ in range(n)]
        pick = [rng.randint(150001, 151000) for _ in range(n)]   # tokens nobody guessed
        at, steps = 0, rng.randint(0, c["depth"])
        for _ in range(steps):
            kids = [j for j in range(max(at + 1, c["depth"] + 1), n) if p[j] == at]
            if not kids:
                break
            at_next = rng.choice(kids)
            pick[at] = tok[at_next]
            at = at_next
        parents += p
        draft += tok
        chosen += pick
    s = dict(case=c, table=_ints(table), len=_ints(lens), refs=_ints(refs), want=_ints(lens),
             first=_ints([n * i for i in range(b + 1)]), parent=_ints(parents), draft=_ints(draft), chosen=_ints(chosen))
    shape = (c["layers"], total, page, c["hk"], c["d"])
    s["pool_k"], s["pool_v"] = _randn(g, shape, dt), _randn(g, shape, dt)
    s["path"] = torch.empty(n * b, dtype=torch.int32, device=DEV)
    s["accepted"] = torch.empty(b, dtype=torch.int32, device=DEV)
    s["next"] = torch.empty(b, dtype=torch.int32, device=DEV)
    return s


def _prepare_w4(c, seed, g, dt):
    n, k, m = c["n"], c["k"], DT[c["meta"]]
    s = dict(case=c)
    s["codes"] = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    unit = 1.0 / (4.6 * math.sqrt(k))                            # outputs of about the size of the inputs
    s["w_scale"] = (unit * (0.5 + torch.rand(n, k // c["group"], generator=g, device=DEV))).to(m)
    s["w_zero"] = None
    if c["zero"]:
        s["w_zero"] = (-unit * (6.5 + 2.0 * torch.rand(n, k // c["group"], generator=g, device=DEV))).to(m)
    s["x"] = _randn(g, (c["rows"], k), dt)
    s["bias"] = _randn(g, (n,), dt) if c["bias"] else None
    s["add"] = _randn(g, (c["rows"], n), dt) if c["add"] else None
    s["y"] = torch.empty(c["rows"], n, dtype=dt, device=DEV)
    return s


def prepare(case, seed):
    g, dt = _gen(seed), DT[case["dtype"]]
    s = {"tree": _prepare_tree, "accept": _prepare_accept, "w4": _prepare_w4}[case["op"]](case, seed, g, dt)
    if own:
        from paper_2510_18269_b200 import oqm
        s["oqm"] = oqm
        if case["op"] == "w4":
            s["w"] = oqm.W4Matrix(s["codes"], s["w_scale"], s["w_zero"])
            return s
        s["pool"] = oqm.KvPool(s["pool_k"], s["pool_v"])
        s["seqs"] = oqm.KvSeqs(s["table"], s["len"], s.get("refs"))
        if case["op"] == "tree":
            need = oqm.stom_kv_attend_tree_workspace_bytes(s["pool"], s["seqs"], s["q"].shape[0], case["hq"])
        else:
            need = oqm.stom_kv_pages_workspace_bytes(s["pool"], s["seqs"])
        s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------- plain forms

def _seen(n, m, window, parent):
    """[m][n] which of n tokens, the last m of them new, each of the new ones sees."""
    base = n - m
    j = torch.arange(m, device=DEV)
    if parent is None:
        on_path = j[None, :] <= j[:, None]
    else:
        # with the parents' rows of ones added until nothing changes: as many doublings as a path of m nodes needs
        on_path = torch.eye(m, dtype=torch.bool, device=DEV)
        step = torch.zeros(m, m, dtype=torch.float32, device=DEV)
        step.scatter_(1, parent.long().clamp(min=0)[:, None], (parent >= 0).float()[:, None])
        reach = on_path.float() + step
        for _ in range(max(1, (m - 1).bit_length())):
            reach = (torch.matmul(reach, reach) > 0).float()
        on_path = reach > 0
    depth = on_path.sum(1) - 1
    place = torch.cat([torch.arange(base, device=DEV), base + depth])          # position of every token
    seen = torch.cat([torch.ones(m, base, dtype=torch.bool, device=DEV), on_path], 1)
    if window:
        seen = seen & (place[None, :] > (base + depth)[:, None] - window)
    return seen


def _run_tree(s):
    c, page, first = s["case"], s["case"]["page"], s["first_host"]
    hk, g = c["hk"], c["hq"] // c["hk"]
    for i, n in enumerate(s["lens"]):
        a, b = first[i], first[i + 1]
        m = b - a
        ids = s["table"][i, :_held(n, page)].long()
        k = s["pool_k"][0][ids].reshape(-1, hk, c["d"])[:n].permute(1, 2, 0).float()
        v = s["pool_v"][0][ids].reshape(-1, hk, c["d"])[:n].permute(1, 0, 2).float()
        q = s["q"][a:b].float().view(m, hk, g, c["d"]).permute(1, 0, 2, 3).reshape(hk, m * g, c["d"])
        x = torch.matmul(q, k) * s["scale"]
        if c["cap"]:
            x = c["cap"] * torch.tanh(x / c["cap"])
        seen = _seen(n, m, c["window"], None if s["parent"] is None else s["parent"][a:b])
        x = x.view(hk, m, g, n).masked_fill_(~seen[None, :, None, :], -math.inf)
        top = x.amax(-1, keepdim=True)
        w = x.sub_(top).exp_()
        z = w.sum(-1, keepdim=True)
        o = torch.matmul(w.view(hk, m * g, n), v).view(hk, m, g, c["d"]) / z
        s["out"][a:b] = o.permute(1, 0, 2, 3).reshape(m, c["hq"], c["d"]).to(s["out"].dtype)
        s["lse"][a:b] = (top + torch.log(z))[..., 0].permute(1, 0, 2).reshape(m, c["hq"])


def _run_accept(s):
    c, table, refs, n = s["case"], s["table"], s["refs"], s["len"]
    page, m, b = c["page"], c["nodes"], c["seqs"]
    cols = torch.arange(table.shape[1], device=DEV)[None, :]
    # room for the drafted tokens: pages of the lowest free ids
    had, new = (n + page - 1) // page, (s["want"] + page - 1) // page
    more = (cols >= had[:, None]) & (cols < new[:, None])
    free = torch.nonzero(refs == 0)[:, 0]
    taken = free[:int(more.sum())]
    table[more] = taken.to(torch.int32)
    refs[taken] = 1
    n.copy_(torch.maximum(n, s["want"]))
    # the walk
    base = n - m
    parent, draft, chosen = s["parent"].view(b, m), s["draft"].view(b, m), s["chosen"].view(b, m)
    at, on = torch.zeros(b, dtype=torch.long, device=DEV), torch.ones(b, dtype=torch.bool, device=DEV)
    path = torch.full((b, m), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = 0
    count = torch.ones(b, dtype=torch.int32, device=DEV)
    node = torch.arange(m, device=DEV)[None, :]
    for k in range(1, c["depth"] + 1):
        fits = (parent == at[:, None]) & (draft == chosen.gather(1, at[:, None])) & (node > at[:, None]) & on[:, None]
        child = torch.where(fits, node, m).amin(1)
        on = child < m
        at = torch.where(on, child, at)
        path[:, k] = torch.where(on, child, -1).to(torch.int32)
        count += on
    s["path"].copy_(path.view(-1))
    s["accepted"].copy_(count)
    s["next"].copy_(chosen.gather(1, at[:, None])[:, 0])
    # the path's keys and values behind the context
    steps = torch.arange(c["depth"] + 1, device=DEV)[None, :]
    to, of = base[:, None] + steps, base[:, None] + path[:, :c["depth"] + 1]
    moves = steps < count[:, None]
    to_page, of_page = (table.long().gather(1, (x // page).long().clamp(0, table.shape[1] - 1))[moves] for x in (to, of))
    to_row, of_row = (to % page)[moves].long(), (of % page)[moves].long()
    for pool in (s["pool_k"], s["pool_v"]):
        pool[:, to_page, to_row] = pool[:, of_page, of_row]
    # lengths, and the pages that are no longer needed
    old, keep = (n + page - 1) // page, (base + count + page - 1) // page
    gone = (cols >= keep[:, None]) & (cols < old[:, None])
    refs.scatter_add_(0, table[gone].long(), torch.full_like(table[gone], -1))
    table.masked_fill_(gone, -1)
    n.copy_(base + count)


def _run_w4(s):
    c = s["case"]
    code = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).view(c["n"], -1, c["group"]).float()
    scale = s["w_scale"].float()[..., None]
    zero = s["w_zero"].float()[..., None] if c["zero"] else scale * -8.0
    w = code.mul_(scale).add_(zero).view(c["n"], c["k"])
    y = torch.matmul(s["x"].float(), w.T)
    if c["bias"]:
        y += s["bias"].float()
    if c["add"]:
        y += s["add"].float()
    s["y"].copy_(y)


def _outputs(s):
    op = s["case"]["op"]
    if op == "tree":
        return [s["out"], s["lse"]]
    if op == "accept":
        return [s["table"], s["len"], s["refs"], s["path"], s["accepted"], s["next"], s["pool_k"], s["pool_v"]]
    return [s["y"]]


def run(state):
    s, c = state, state["case"]
    if not own:
        {"tree": _run_tree, "accept": _run_accept, "w4": _run_w4}[c["op"]](s)
    elif c["op"] == "tree":
        s["oqm"].stom_kv_attend_tree(s["pool"], s["seqs"], 0, s["first"], s["q"], s["out"], s["scale"], s["ws"],
                                     parent=s["parent"], lse=s["lse"], softcap=c["cap"], window=c["window"])
    elif c["op"] == "accept":
        s["oqm"].stom_kv_reserve(s["pool"], s["seqs"], s["want"], s["ws"])
        s["oqm"].stom_kv_accept(s["pool"], s["seqs"], s["first"], s["draft"], s["chosen"], s["path"], s["accepted"], s["next"],
                                parent=s["parent"])
    else:
        s["oqm"].stom_w4_linear(s["w"], s["x"], s["y"], bias=s["bias"], add=s["add"])
    return _outputs(s)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "tree":
        lens, new, _ = _lens(c, 0)
        e = ESIZE[c["dtype"]]
        kv = pairs = 0
        for n, m in zip(lens, new):
            base = n - m
            w = c["window"] or n
            kv += min(n, w + m) * c["hk"] * c["d"] * 2 * e
            pairs += m * min(base + (m + 1) // 2, w) if c["shape"] != "tree" else m * min(base + 1, w)
        rows = sum(new) * c["hq"]
        return {"bytes": kv + rows * (c["d"] * 2 * e + 4), "flops": 4 * pairs * c["hq"] * c["d"]}
    if c["op"] == "accept":
        moved = c["seqs"] * (c["depth"] / 2.0) * c["layers"] * c["hk"] * c["d"] * 2 * ESIZE[c["dtype"]]
        return {"bytes": int(2 * moved) + c["seqs"] * c["nodes"] * 16, "flops": 0}
    meta = c["n"] * (c["k"] // c["group"]) * ESIZE[c["meta"]] * (2 if c["zero"] else 1)
    e = ESIZE[c["dtype"]]
    rest = (c["rows"] * (c["k"] + c["n"] * (2 if c["add"] else 1)) + (c["n"] if c["bias"] else 0)) * e
    return {"bytes": c["n"] * c["k"] // 2 + meta + rest, "flops": 2 * c["rows"] * c["n"] * c["k"]}


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _exact_tree(s):
    c, page = s["case"], s["case"]["page"]
    g = c["hq"] // c["hk"]
    first = s["first"].tolist()
    parent = None if s["parent"] is None else s["parent"].tolist()
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for i, n in enumerate(s["len"].tolist()):
        m = first[i + 1] - first[i]
        base = n - m
        t = torch.arange(n, device=DEV)
        ids = s["table"][i].long()[t // page]
        # rows of what is hidden, node by node
        depth, hidden = [], torch.ones(m, n, dtype=torch.bool)
        for j in range(m):
            p = j - 1 if parent is None else parent[first[i] + j]
            depth.append(0 if p < 0 else depth[p] + 1)
            if p >= 0:
                hidden[j, base:] = hidden[p, base:]
            hidden[j, :base] = False
            hidden[j, base + j] = False
        if c["window"]:
            place = torch.tensor(list(range(base)) + [base + x for x in depth])
            hidden |= place[None, :] <= place[base:, None] - c["window"]
        hidden = hidden.to(DEV)
        for h in range(c["hk"]):
            k, v = s["pool_k"][0, ids, t % page, h].double(), s["pool_v"][0, ids, t % page, h].double()
            for a in range(0, m, 256):
                z = slice(first[i] + a, first[i] + min(m, a + 256))
                x = torch.einsum("jgd,td->gjt", s["q"][z, h * g:(h + 1) * g].double(), k) * s["scale"]
                if c["cap"]:
                    x = torch.tanh(x / c["cap"]) * c["cap"]
                x.masked_fill_(hidden[None, a:a + 256], -math.inf)
                lse[z, h * g:(h + 1) * g] = torch.logsumexp(x, -1).T
                out[z, h * g:(h + 1) * g] = torch.einsum("gjt,td->jgd", torch.softmax(x, -1), v)
    return [out, lse]


def _exact_accept(s):
    c = s["case"]
    page, m = c["page"], c["nodes"]
    table, n, refs = s["table"].tolist(), s["len"].tolist(), s["refs"].tolist()
    parent, draft, chosen = s["parent"].tolist(), s["draft"].tolist(), s["chosen"].tolist()
    path, accepted, following = [], [], []
    for i in range(c["seqs"]):
        base, z = n[i] - m, i * m
        way = [0]
        while True:
            kids = [j for j in range(m) if parent[z + j] == way[-1] and draft[z + j] == chosen[z + way[-1]]]
            if not kids:
                break
            way.append(kids[0])
        for pool in (s["pool_k"], s["pool_v"]):
            for k, j in enumerate(way):
                a, o = base + k, base + j
                pool[:, table[i][a // page], a % page] = pool[:, table[i][o // page], o % page]
        for j in range(_held(base + len(way), page), _held(n[i], page)):
            refs[table[i][j]] -= 1
            table[i][j] = -1
        n[i] = base + len(way)
        path += way + [-1] * (m - len(way))
        accepted.append(len(way))
        following.append(chosen[z + way[-1]])
    return [_ints(table), _ints(n), _ints(refs), _ints(path), _ints(accepted), _ints(following), s["pool_k"], s["pool_v"]]


def _exact_w4(s):
    c = s["case"]
    x = s["x"].double()
    y = torch.empty(c["rows"], c["n"], dtype=torch.float64, device=DEV)
    for a in range(0, c["n"], 8192):
        codes = s["codes"][a:a + 8192].long()
        w = torch.empty(codes.shape[0], c["k"], dtype=torch.float64, device=DEV)
        w[:, 0::2], w[:, 1::2] = (codes % 16).double(), (codes // 16).double()
        scale = s["w_scale"][a:a + 8192].double().repeat_interleave(c["group"], 1)
        w = w * scale + s["w_zero"][a:a + 8192].double().repeat_interleave(c["group"], 1) if c["zero"] else (w - 8) * scale
        y[:, a:a + 8192] = x @ w.T
    if c["bias"]:
        y = y + s["bias"].double()
    if c["add"]:
        y = y + s["add"].double()
    return [y]


def exact(case, seed):
    global own
    was, own = own, False                                        # inputs only
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"tree": _exact_tree, "accept": _exact_accept, "w4": _exact_w4}[case["op"]](s)
