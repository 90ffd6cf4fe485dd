"""How exact the softmax weights of stom_kv_attend_tree are: as exact as those of a single token's attention.

Tolerance of out, element by element, with u the type's half step (2^-8 bf16, 2^-11 fp16):
    u |out|                         the one rounding of the result
  + mean_w|V| * (2 u^2 + 2^-15)     a weight's low part is rounded to u of itself (u^2 of the weight, with a factor 2 for the
                                    subtraction); scores, exponentials and sums in binary32: scores below 32 in magnitude
                                    carry below 2^-16 from their sum and scaling, the exponential doubles it at most
  + 2^-24 + 2^-32 n max|V| (fp16)   where the result is subnormal; a low part below fp16's smallest step is off by half of it,
                                    2^-25 where the row's largest weight is 2^7 or more, for each of n tokens (their weights
                                    relative to the largest sum to 1 at least)"""
import numpy as np
import pytest
import torch

import _kv as K
import _tree as T
from test_gpu_kv_tree import BF, HF, _call, _make

pytestmark = pytest.mark.gpu


def _close(s, out, scale, cap=0.0, window=0):
    n, dtype = s["first"][-1], out.dtype
    want, wlse, mag = T.attend_nodes(s["k"], s["v"], s["table_host"], s["lens"], s["first"], s["parent"], s["q"], scale, cap, window)
    assert np.abs(wlse[:n][np.isfinite(wlse[:n])]).max(initial=0.0) < 32
    u = K.HALF_STEP[dtype]
    lim = u * np.abs(want) + mag * (2 * u * u + 2.0 ** -15)
    if dtype is HF:
        lim = lim + 2.0 ** -24 + 2.0 ** -32 * max(s["lens"]) * s["v"].abs().max().item()
    off = np.abs(out.double().cpu().numpy() - want)[:n]
    assert (off <= lim[:n]).all(), (int((off > lim[:n]).sum()), float(np.max(off / lim[:n])))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("had,new,hq,hk,d,page,kind,cap,window", [
    ([12583], [5], 28, 4, 128, 50, "path", 0.0, 0),        # one stream over the whole device
    ([2500], [64], 28, 4, 128, 50, "tree", 0.0, 0),
    ([333, 64, 129], [20, 19, 18], 16, 2, 64, 1, "forest", 0.0, 0),
    ([300, 77, 5, 0], [40, 1, 9, 3], 8, 4, 256, 16, "tree", 0.0, 0),
    ([1000, 0, 77], [129, 300, 1], 14, 2, 128, 50, "chain", 0.0, 0),
    ([64], [211], 3, 3, 256, 64, "chain", 0.0, 100),
    ([250, 0, 130, 3], [20, 9, 1, 40], 8, 2, 128, 16, "tree", 20.0, 100),
    ([700, 3], [13, 20], 12, 1, 64, 7, "roots", 30.0, 0),
])
def test_weights_lose_nothing_that_shows(dtype, had, new, hq, hk, d, page, kind, cap, window):
    s = _make(had, new, hq, hk, d, page, dtype, kind)
    out, _ = _call(s, cap=cap, window=window)
    _close(s, out, d ** -0.5, cap, window)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_weights_all_alike(dtype):
    """Many tokens of the same weight, values of either sign that all but cancel: an error of the weights would show whole."""
    s = _make([4000], [3], 4, 2, 128, 50, dtype, "path")
    s["k"].zero_()
    s["k"][..., 0] = torch.arange(50, device="cuda").to(dtype)[:, None] / 32   # weights that are no powers of two
    s["q"].zero_()
    s["q"][..., 0] = 1.0
    out, _ = _call(s, scale=0.7)
    _close(s, out, 0.7)
