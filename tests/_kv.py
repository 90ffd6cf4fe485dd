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
