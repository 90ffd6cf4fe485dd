"""Plain implementations in 64 bits that the tests of the paged cache and of the token choice compare with, and the
builders of their inputs.  Written from the formulas in include/stom_kv.h and include/stom_sample.h, row by row."""
import math

import numpy as np
import torch

#: the largest relative error of one rounding to the type
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def paged(rng, lens, page, layers, heads, d, dtype, spare=3, order="token", width=None, seed=0):
    """A pool of shuffled pages for these lengths: dict of tensors on the GPU.  order: which of token and head is the
    outer axis of a page."""
    held = [-(-n // page) for n in lens]
    total = sum(held) + spare
    ids = rng.permutation(total)[:sum(held)]
    width = width or max([1] + held)
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    refs = np.zeros(total, np.int32)
    for i, m in enumerate(held):
        table[i, :m] = ids[at:at + m]
        refs[ids[at:at + m]] = 1
        at += m
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (layers, total, page, heads, d) if order == "token" else (layers, total, heads, page, d)
    k, v = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
    if order == "head":
        k, v = k.permute(0, 1, 3, 2, 4), v.permute(0, 1, 3, 2, 4)
    dev = dict(table=torch.from_numpy(table).cuda(), len=torch.tensor(lens, dtype=torch.int32, device="cuda"),
               refs=torch.from_numpy(refs).cuda())
    return dict(k=k, v=v, table_host=table, **dev)


def attend_rows(pool_k, pool_v, table, lens, q, scale, cap=0.0, window=0, layer=0):
    """out, lse, and the softmax-weighted mean of |V| (what an error of the weights is relative to), float64 on the CPU."""
    n, hq, d = q.shape
    _, pages, page, hk, _ = pool_k.shape
    g = hq // hk
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    mag = np.zeros((n, hq, d))
    qd = q.double().cpu().numpy()
    kd, vd = pool_k[layer].double().cpu().numpy(), pool_v[layer].double().cpu().numpy()
    for i in range(n):
        length = min(max(int(lens[i]), 0), table.shape[1] * page)
        first = max(0, length - window) if window else 0
        t = np.arange(first, length)
        pid = table[i][t // page] if len(t) else t
        good = (pid >= 0) & (pid < pages)
        t, pid = t[good], pid[good]
        if not len(t):
            continue
        for h in range(hq):
            x = kd[pid, t % page, h // g] @ qd[i, h] * scale
            if cap:
                x = cap * np.tanh(x / cap)
            top = x.max()
            w = np.exp(x - top)
            lse[i, h] = top + math.log(w.sum())
            rows = vd[pid, t % page, h // g]
            out[i, h] = w @ rows / w.sum()
            mag[i, h] = w @ np.abs(rows) / w.sum()
    return out, lse, mag


def turned(x, pos, freq, layout, weight=None, eps=1e-6, magnitude=1.0):
    """Norm and rotation of [n][heads][d], float64 on the CPU; and a bound on the magnitude of the terms of an element."""
    y = x.double().cpu().numpy().copy()
    if weight is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps) * weight.double().cpu().numpy()
    mag = np.abs(y)
    f = freq.double().cpu().numpy()
    h = len(f)
    angle = pos.cpu().numpy().astype(np.float64)[:, None] * f[None, :]
    c, s = (np.cos(angle) * magnitude)[:, None, :], (np.sin(angle) * magnitude)[:, None, :]
    ia = np.arange(h) if layout == 0 else 2 * np.arange(h)
    ib = ia + h if layout == 0 else ia + 1
    a, b = y[..., ia].copy(), y[..., ib].copy()
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    m = abs(magnitude) * (np.abs(a) + np.abs(b))
    mag[..., ia], mag[..., ib] = m, m
    return y, mag


class Book:
    """The pages of a cache kept in Python, one rule after the other, for what the device decides in parallel."""

    def __init__(self, table, lens, refs, page, k, v):
        self.table, self.len, self.refs, self.page = table.copy(), list(lens), refs.copy(), page
        self.k, self.v = k.clone(), v.clone()

    def held(self, n):
        return -(-n // self.page)

    def free(self, drop):
        for i, gone in enumerate(drop):
            if gone:
                for j in range(self.held(self.len[i])):
                    self.refs[self.table[i, j]] -= 1
                self.table[i], self.len[i] = -1, 0

    def fork(self, parent):
        before = list(self.len)
        for i, f in enumerate(parent):
            if f >= 0 and parent[f] == -1 and before[i] == 0:
                m = self.held(before[f])
                self.table[i] = -1
                self.table[i, :m] = self.table[f, :m]
                self.len[i] = before[f]
                for j in range(m):
                    self.refs[self.table[f, j]] += 1

    def reserve(self, want):
        keep = (self.table.copy(), list(self.len), self.refs.copy(), self.k.clone(), self.v.clone())
        free = [p for p, r in enumerate(self.refs) if r == 0]
        try:
            for i, w in enumerate(want):
                n = self.len[i]
                if w <= n or w > self.table.shape[1] * self.page:
                    continue
                m = self.held(n)
                if n % self.page and self.refs[self.table[i, m - 1]] > 1:
                    old, new = self.table[i, m - 1], free.pop(0)
                    self.refs[old] -= 1
                    self.refs[new], self.table[i, m - 1] = 1, new
                    for x in (self.k, self.v):
                        x[:, new, :n % self.page] = x[:, old, :n % self.page]
                for j in range(m, self.held(w)):
                    self.table[i, j] = free.pop(0)
                    self.refs[self.table[i, j]] = 1
                self.len[i] = w
            return True
        except IndexError:                                       # out of pages: as if nothing had been asked
            self.table, self.len, self.refs, self.k, self.v = keep
            return False

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = [p for p in range(live) if self.refs[p] <= 0]
        for p in range(live, len(self.refs)):
            if self.refs[p] > 0:
                to = holes.pop(0)
                for x in (self.k, self.v):
                    x[:, to] = x[:, p]
                self.refs[to], self.refs[p] = self.refs[p], 0
                self.table[self.table == p] = to
        return live


def choose(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(acceptable tokens, acceptable counts, {token: logprob}) of one row by sorting it, in 64 bits.  More than one is
    acceptable only where a mass comes within NEAR of the border asked for."""
    x = np.asarray(x, np.float64)
    order = np.argsort(-np.where(np.isnan(x), -np.inf, x) + 0.0, kind="stable")
    order = order[~np.isnan(x[order]) & (x[order] > -np.inf)]
    if not len(order):
        return {-1}, {0}, {-1: -np.inf}
    if temperature <= 0:
        return {int(order[0])}, {1}, {int(order[0]): 0.0}
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        y = np.where(x[order] == x[order[0]], 0.0, (x[order] - x[order[0]]) / temperature)
        w = np.where(y < -700.0, 0.0, np.exp(y))
    order, w = order[w > 0], w[w > 0]
    if top_k > 0:
        order, w = order[:top_k], w[:top_k]
    upto = np.cumsum(w)
    near = NEAR * upto[-1]
    counts = {len(w)}
    if top_p < 1:
        aim = max(top_p, 0.0) * upto[-1]
        counts = {int(np.searchsorted(upto, aim + s * near, side="left")) + 1 for s in (-1, 0, 1)}
        exact = aim == upto
        if exact.any():                                          # a tie that both sides can form exactly
            counts = {int(np.argmax(exact)) + 1}
    stay = int((w >= min(min_p, 1.0)).sum())
    counts = {max(1, min(c, stay, len(w))) for c in counts}
    tokens, logprobs = set(), {}
    for c in counts:
        for s in (0,) if (u * upto[c - 1] == upto[:c]).any() else (-1, 0, 1):
            j = int(np.searchsorted(upto[:c], u * upto[c - 1] + s * near * (u > 0), side="right"))
            j = min(j, c - 1)
            tokens.add(int(order[j]))
            logprobs[int(order[j])] = math.log(w[j]) - math.log(upto[c - 1])
    return tokens, counts, logprobs


#: relative error of the masses: 4 096 ranges of masses rounded to 2^-45 of the largest weight, or 131 072 logits each
#: rounded so whose errors add up at random (factor 4 * 362 * 2^-45 = 4e-11), against 150 000 binary64 additions here
NEAR = 1e-10
