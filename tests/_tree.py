"""Plain implementations in 64 bits of attention of several new tokens per sequence, of the acceptance of a drafted path and
of products with 4-bit weights, from the formulas in include/stom_kv.h and include/stom_w4.h; and trees to try them on."""
import math

import numpy as np


def a_tree(rng, n, kind):
    """Parents of n nodes.  kind: "path", "roots" (all follow the context), "star" (all follow node 0), "tree", "forest"."""
    if kind == "path":
        return list(range(-1, n - 1))
    if kind == "roots":
        return [-1] * n
    if kind == "star":
        return [-1] + [0] * (n - 1) if n else []
    low = -1 if kind == "forest" else 0
    return [-1 if j == 0 else int(rng.integers(low, j)) for j in range(n)]


def sees(base, parents, window):
    """Per node, the tokens it sees (ascending): the context's, then those of its path."""
    n = len(parents)
    depth, paths, out = [], [], []
    for j, p in enumerate(parents):
        p = p if -1 <= p < j else -1
        depth.append(depth[p] + 1 if p >= 0 else 0)
        paths.append((paths[p] if p >= 0 else []) + [j])
    for j in range(n):
        at = base + depth[j]
        context = range(max(0, at - window + 1) if window else 0, base)
        nodes = [base + c for c in paths[j] if not window or base + depth[c] > at - window]
        out.append(np.array(list(context) + nodes, dtype=np.int64))
    return out


def attend_nodes(pool_k, pool_v, table, lens, first, parent, q, scale, cap=0.0, window=0, layer=0):
    """out, lse and the softmax-weighted mean of |V| of all rows of q (rows of no sequence: NaN), float64 on the CPU.
    Rows with a token that is not finite are computed without a warning, and come out as the formula has them."""
    rows, hq, d = q.shape
    _, pages, page, hk, _ = pool_k.shape
    g = hq // hk
    out, lse, mag = (np.full(s, np.nan) for s in ((rows, hq, d), (rows, hq), (rows, hq, d)))
    qd = q.double().cpu().numpy()
    kd, vd = pool_k[layer].double().cpu().numpy(), pool_v[layer].double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        for i, length in enumerate(lens):
            a, n = first[i], first[i + 1] - first[i]
            base = length - n
            par = [j - 1 for j in range(n)] if parent is None else list(parent[a:a + n])
            for j, t in enumerate(sees(base, par, window)):
                t = t[t < table.shape[1] * page]
                pid = table[i][t // page] if len(t) else t
                good = (pid >= 0) & (pid < pages)
                t, pid = t[good], pid[good]
                out[a + j], lse[a + j], mag[a + j] = 0.0, -np.inf, 0.0
                if not len(t):
                    continue
                for h in range(hq):
                    x = kd[pid, t % page, h // g] @ qd[a + j, h] * scale
                    if cap:
                        x = cap * np.tanh(x / cap)
                    top = x.max()
                    w = np.exp(x - top)
                    v = vd[pid, t % page, h // g]
                    lse[a + j, h] = top + math.log(w.sum())
                    out[a + j, h] = w @ v / w.sum()
                    mag[a + j, h] = w @ np.abs(v) / w.sum()
    return out, lse, mag


def accept(book, first, parent, draft, chosen):
    """Walks and moves in a Book of _kv; (path, n_accepted, next)."""
    path, counts, following = np.full(first[-1], -1, np.int32), [], []
    for i in range(len(book.len)):
        a, n = first[i], first[i + 1] - first[i]
        if n == 0:
            counts.append(0)
            following.append(-1)
            continue
        base, at, way = book.len[i] - n, 0, [0]
        while chosen[a + at] >= 0:
            kids = [c for c in range(at + 1, n) if (c - 1 if parent is None else parent[a + c]) == at
                    and draft[a + c] == chosen[a + at]]
            if not kids:
                break
            at = kids[0]
            way.append(at)
        for k, j in enumerate(way):
            to, of = base + k, base + j
            for x in (book.k, book.v):
                x[:, book.table[i, to // book.page], to % book.page] = x[:, book.table[i, of // book.page], of % book.page].clone()
        for j in range(book.held(base + len(way)), book.held(book.len[i])):
            book.refs[book.table[i, j]] -= 1
            book.table[i, j] = -1
        book.len[i] = base + len(way)
        path[a:a + len(way)] = way
        counts.append(len(way))
        following.append(int(chosen[a + at]))
    return path, np.array(counts), np.array(following)


def weights(codes, scale, zero, group):
    """[n][k] in 64 bits; codes, scale, zero on the CPU."""
    c = codes.numpy()
    w = np.empty((c.shape[0], 2 * c.shape[1]))
    w[:, 0::2], w[:, 1::2] = c & 15, c >> 4
    s = np.repeat(scale.double().numpy(), group, 1)
    return (w - 8) * s if zero is None else w * s + np.repeat(zero.double().numpy(), group, 1)
