"""Attention of several new tokens where few look: values that are no finite numbers at every head size, in trees and in chains of
several row tiles, with blocks that go through many tiles; sequences out of order; scores of any size."""
import math

import numpy as np
import pytest
import torch

import _kv as K
import _tree as T
from test_gpu_kv_tree import BF, HF, _call, _check, _make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("kind,window", [("tree", 0), ("tree", 70), ("chain", 0), ("chain", 70)])
@pytest.mark.parametrize("d,page,dtype", [(64, 16, BF), (64, 50, HF), (128, 50, HF), (128, 16, BF), (256, 16, BF), (256, 7, HF)])
def test_values_that_are_no_numbers(d, page, dtype, kind, window, value):
    """60 sequences, so that every block goes round its ring; one node of each is spoilt, in one channel of one kv head."""
    rng = np.random.default_rng(d + page)
    had, new = rng.integers(0, 1200, 60).tolist(), rng.integers(1, 45, 60).tolist()
    hq, hk, g = 14, 2, 7
    s = _make(had, new, hq, hk, d, page, dtype, kind, seed=d)
    want = _call(s, window=window)
    seen, blind = [], torch.ones(s["rows"], dtype=torch.bool)
    spoilt = []
    for i, n in enumerate(new):
        j, a = int(rng.integers(0, n)), s["first"][i]
        parents = [x - 1 for x in range(n)] if kind == "chain" else s["parent"][a:a + n]
        rows = [a + b for b, tokens in enumerate(T.sees(had[i], parents, window)) if had[i] + j in tokens]
        seen += rows
        blind[rows] = False
        spoilt.append((int(s["table_host"][i, (had[i] + j) // page]), (had[i] + j) % page))
    blind = blind.cuda()
    others = torch.ones(d, dtype=torch.bool, device="cuda")
    others[5] = False
    for name in ("k", "v"):
        keep = s[name].clone()
        for page_id, slot in spoilt:
            s[name][0, page_id, slot, 1, 5] = value
        out, lse = _call(s, window=window)
        s[name].copy_(keep)
        assert torch.equal(out[blind], want[0][blind]) and torch.equal(lse[blind], want[1][blind])
        assert torch.equal(out[:, :g], want[0][:, :g]) and torch.equal(lse[:, :g], want[1][:, :g])   # heads of the other kv head
        if name == "v":
            assert not torch.isfinite(out[seen][:, g:, 5]).any()
            assert torch.equal(out[..., others], want[0][..., others]) and torch.equal(lse, want[1])


def test_sequences_out_of_order():
    """The second begins behind its end: it is skipped and flagged, the others, whose rows do not meet, are right."""
    s = _make([50, 300, 60], [0, 2, 11], 4, 2, 64, 16, BF, "tree", extra=6)
    t = dict(s, first=[6, 6, 4, 15], parent=[-1] * 4 + s["parent"][2:13])
    t["q"] = torch.cat([s["q"][-4:], s["q"][2:13], s["q"][13:17]])
    out, lse = _call(t, flag=1)
    want, wlse, mag = T.attend_nodes(s["k"], s["v"], s["table_host"][2:], [71], [0, 11], s["parent"][2:13], t["q"][4:15], 64 ** -0.5)
    u = K.HALF_STEP[BF]
    off = np.abs(out[4:15].double().cpu().numpy() - want)
    assert (off <= u * np.abs(want) + mag * (2 * u * u + 2.0 ** -15)).all()
    assert (np.abs(lse[4:15].double().cpu().numpy() - wlse) <= 2.0 ** -15 + 2.0 ** -22 * np.abs(wlse)).all()
    assert (out[:4] == 7.0).all() and (out[15:] == 7.0).all() and (lse[:4] == 7.0).all() and (lse[15:] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("scale", [5.0, 50.0, -50.0])
def test_large_scores(scale, d, dtype):
    """A score's error is that of its binary32 sum and scaling, below 2^-21 |q| |k| |scale| (2^-16 where that is 32): it changes a
    weight by as much, relatively, and the sum that it is divided by once more."""
    s = _make([500, 20], [33, 4], 4, 2, d, 16, dtype)
    out, lse = _call(s, scale=scale)
    n = s["first"][-1]
    want, wlse, mag = T.attend_nodes(s["k"], s["v"], s["table_host"], s["lens"], s["first"], s["parent"], s["q"], scale)
    most = abs(scale) * s["q"].double().norm(dim=-1).max().item() * s["k"].double().norm(dim=-1).max().item()
    off, u = 2.0 ** -21 * most, K.HALF_STEP[dtype]
    lim = u * np.abs(want) + mag * (2 * u * u + 2 * off) + (2.0 ** -24 + 2.0 ** -32 * 533 * 6 if dtype is HF else 0)
    assert (np.abs(out[:n].double().cpu().numpy() - want[:n]) <= lim[:n]).all()
    assert (np.abs(lse[:n].double().cpu().numpy() - wlse[:n]) <= off + 2.0 ** -22 * np.abs(wlse[:n])).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("scale", [1e30, -1e30])
def test_scores_near_the_largest_number(scale, dtype):
    """Nothing but the largest score counts."""
    s = _make([500, 20], [33, 4], 4, 2, 128, 16, dtype)
    out, lse = _call(s, scale=scale)
    kd, qd, page = s["k"][0].double().cpu().numpy(), s["q"].double().cpu().numpy(), 16
    compared = 0
    for i, length in enumerate(s["lens"]):
        a, b = s["first"][i], s["first"][i + 1]
        for j, t in enumerate(T.sees(length - (b - a), s["parent"][a:b], 0)):
            pid = s["table_host"][i][t // page]
            for h in range(4):
                x = np.sign(scale) * (kd[pid, t % page, h // 2] @ qd[a + j, h])
                top = int(np.argmax(x))
                if x[top] - np.delete(x, top).max(initial=-np.inf) > 2.0 ** -10:        # (a sum of 128 products is off by 2^-16)
                    assert torch.equal(out[a + j, h], s["v"][0, pid[top], t[top] % page, h // 2])
                    assert abs(lse[a + j, h].item() / (abs(scale) * x[top]) - 1) < 2.0 ** -20
                    compared += 1
    assert compared > 100


def test_a_scale_near_nothing():
    s = _make([500, 20], [33, 4], 4, 2, 128, 16, BF)
    _check(s, *_call(s, scale=1e-30), scale=1e-30)
