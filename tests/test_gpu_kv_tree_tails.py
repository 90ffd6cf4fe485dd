"""stom_kv_attend_tree in fp16 where tokens count only in sum beside one that stands far above them, with a value of zero: the
result is theirs alone, however little each of them weighs.

Tolerance of out, with w the weights relative to the row's largest, u = 2^-11:
    u |out| + mean_w|V| * (2 u^2 + 2^-15)    as where no weight is small
  + 2^-24                                    where the result is subnormal
  + sum_t e_t |V_t| / sum_t w_t              e_t: a weight's low part is off by half of fp16's smallest step, 2^-25, where the
                                             weight of the reference is 2^7: 2^-32 of the largest weight so far, and at most
                                             2^-24 of the largest of its own tile's, one of the 127 tokens on either side"""
import numpy as np
import pytest
import torch

import _kv as K
from test_gpu_kv_tree import BF, HF, _call, _close_lse, _make

pytestmark = pytest.mark.gpu


def _check(had, new, hq, hk, d, page, scores, silent, dtype=HF, window=0):
    """scores: of every token of each sequence (nodes too, one after another); silent: tokens whose value is zero."""
    s = _make(had, new, hq, hk, d, page, dtype, "chain")
    s["k"].zero_()
    s["v"].copy_(s["v"].abs() + 0.25)
    for i, x in enumerate(scores):
        t = np.arange(len(x))
        at = torch.from_numpy(s["table_host"][i, t // page]).long().cuda(), torch.from_numpy(t % page).cuda()
        s["k"][0, at[0], at[1], :, 0] = torch.from_numpy(x).to(dtype).cuda()[:, None]
        z = torch.from_numpy(np.asarray(silent[i])).cuda()
        s["v"][0, at[0][z], at[1][z]] = 0
    s["q"].zero_()
    s["q"][..., 0] = 4.0                                           # times a scale of 0.25: the score is the key's entry
    out, lse = _call(s, scale=0.25, window=window)
    got, u = out.double().cpu().numpy(), K.HALF_STEP[dtype]
    for i, x in enumerate(scores):
        t = np.arange(len(x))
        x = s["k"][0, s["table_host"][i, t // page], t % page, 0, 0].double().cpu().numpy()
        v = s["v"][0, s["table_host"][i, t // page], t % page].double().cpu().numpy()       # [token][head][channel]
        for j in range(new[i]):
            end = had[i] + j + 1
            begin = max(0, end - window) if window else 0
            w = np.exp(x[begin:end] - x[begin:end].max())
            reach = np.pad(w, 127)
            near = np.max(np.lib.stride_tricks.sliding_window_view(reach, 255), axis=1)
            e = np.minimum(2.0 ** -32, 2.0 ** -24 * near) if dtype is HF else 0 * w
            row = s["first"][i] + j
            _close_lse(lse[row], np.full(hq, x[begin:end].max() + np.log(w.sum())))
            for h in range(hq):
                y = v[begin:end, h // (hq // hk)]
                want = w @ y / w.sum()
                lim = u * want + want * (2 * u * u + 2.0 ** -15) + (2.0 ** -24 if dtype is HF else 0) + e @ y / w.sum()
                off = np.abs(got[row, h] - want)
                assert (off <= lim).all(), (i, j, h, float(np.max(off / lim)))


def _sink(n, gap, at):
    x, silent = np.zeros(n), np.zeros(n, bool)
    x[at], silent[at] = gap, True
    return x, silent


@pytest.mark.parametrize("gap", [4.0, 10.0, 15.5, 17.0, 20.0, 24.0])
@pytest.mark.parametrize("had,new,hq,hk,d,page", [
    ([12583], [5], 2, 1, 128, 50),                       # one unit over all blocks
    ([600] * 60, [3] * 60, 2, 1, 64, 50),                # units of a few tiles
    ([5000, 40], [40, 9], 12, 1, 128, 7),                # several row tiles
    ([3000, 17], [2, 30], 1, 1, 256, 16),
])
def test_a_tail_beside_one_token(had, new, hq, hk, d, page, gap):
    both = [_sink(a + b, gap, min(3, a - 1)) for a, b in zip(had, new)]
    _check(had, new, hq, hk, d, page, [x for x, _ in both], [z for _, z in both])


@pytest.mark.parametrize("n,gap", [(131072, 20.0), (131072, 24.0), (400009, 22.5)])
def test_a_long_tail(n, gap):
    x, silent = _sink(n + 2, gap, n // 2)
    _check([n], [2], 1, 1, 64, 64, [x], [silent])


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 3000])
def test_references_that_fall_and_rise(d, window):
    """Every 300th token far above its neighbours; and scores that go down by 40 in all, and up again."""
    n = 6000
    x, silent = np.zeros(n + 3), np.zeros(n + 3, bool)
    x[5::300], silent[5::300] = 14.0, True
    down = -np.arange(n + 3) / (n / 40.0)
    # what is above the tail's -25 is silent, so that the tail is the result
    _check([n] * 3, [3] * 3, 2, 1, d, 50, [x, down, down[::-1].copy()], [silent, down > -25, down[::-1] > -25], window=window)


def test_a_tail_too_far_below_to_show():
    """Scores hundreds below the largest: their weights are zeros, nothing overflows."""
    s = _make([3000], [2], 2, 1, 64, 50, HF, "chain")
    s["k"].zero_()
    s["k"][0, s["table_host"][0, 0], 40, :, 0] = 600.0
    s["q"].zero_()
    s["q"][..., 0] = 4.0
    out, lse = _call(s, scale=0.25)
    assert torch.equal(out[0, 0], s["v"][0, s["table_host"][0, 0], 40, 0]) and torch.equal(out[1], out[0])
    assert (lse - 600.0).abs().max().item() <= 600 * 2.0 ** -22


def test_bf16_has_the_exponents():
    x, silent = _sink(12588, 24.0, 3)
    _check([12583], [5], 2, 1, 128, 50, [x], [silent], dtype=BF)
