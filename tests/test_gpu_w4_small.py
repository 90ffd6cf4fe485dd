"""Values of a token far below the largest of their group in the products with 4-bit weights, by the bounds that include/stom_w4.h
gives: nothing is lost down to 2^-24 (fp16) or 2^-27 (bf16) of the largest, and below 2^-35 of the largest at most."""
import math

import pytest
import torch

from test_gpu_w4 import BF, HF, _lib

pytestmark = pytest.mark.gpu


def _products(rows, small, top, dtype, columns, group, alike):
    """The largest value of every group meets a code of 0, all others, at `columns` of every eight, codes 1 to 15: the sums are
    of the small values alone, which are all alike (as are their roundings then) or one or three times as large.  Result, the
    sums in 64 bits, and the sums of the codes."""
    oqm = _lib()
    n, k = 40, 4 * group
    g = torch.Generator().manual_seed(1)
    code = torch.randint(1, 16, (n, k), generator=g)
    code[:, ::group] = 0
    x = torch.zeros(rows, k, dtype=torch.float64)
    for c in columns:
        x[:, c::8] = small * (1 if alike else 1 + torch.randint(0, 2, (rows, k // 8), generator=g).double() * 2)
    x[:, ::group] = top
    x = x.to(dtype)
    packed = (code[:, 0::2] | code[:, 1::2] << 4).to(torch.uint8).cuda()
    scale = torch.ones(n, k // group, dtype=torch.float32, device="cuda")
    power = 2.0 ** (-6 - math.floor(math.log2(small)))             # exact, and the results are some ten or hundred
    y = torch.empty(rows, n, dtype=dtype, device="cuda")
    oqm.stom_w4_linear(oqm.W4Matrix(packed, scale * power, torch.zeros_like(scale)), x.cuda(), y)
    torch.cuda.synchronize()
    want = (x.double() @ code.double().T) * power
    seen = x.double() != 0
    seen[:, ::group] = False
    return y.double().cpu(), want, (seen.double() @ code.double().T) * power


@pytest.mark.parametrize("rows", [1, 8, 20, 64])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("alike", [True, False])
@pytest.mark.parametrize("columns", [(1, 3, 5, 7), (2, 4, 6), (1, 2, 3, 4, 5, 6, 7)])
@pytest.mark.parametrize("dtype,top", [(BF, 1.0), (BF, 1.75), (HF, 2.0 ** 15), (HF, 2.0 ** 15 * 1.75)])
def test_small_values_beside_a_large_one(rows, group, columns, alike, dtype, top):
    u = 2.0 ** -8 if dtype is BF else 2.0 ** -11
    least = 2.0 ** (-27 if dtype is BF else -24)
    whole = 2.0 - 2.0 ** (-7 if dtype is BF else -10)                                # all bits set
    one = 2.0 ** (0 if dtype is BF else 15)
    for small in (whole * least * one * 2, 1.5 * 2.0 ** -34 * one, 1.25 * 2.0 ** -33 * one, 2.0 ** -36 * one):
        got, want, codes = _products(rows, small, top, dtype, columns, group, alike)
        lost = 0.0 if small >= least * top else 2.0 ** -35 * top
        # what small values lose, sums in binary32 of up to 128 a group, and the rounding of the result: it is one of what
        # has been lost from, |y'| <= |want| + lost * codes, so that (1 + u) lost * codes stands for both
        lim = (u + 2.0 ** -16) * want.abs() + (1 + u) * lost * codes + (2.0 ** -24 if dtype is HF else 0)
        assert ((got - want).abs() <= lim).all(), (small, float(((got - want).abs() / lim).max()))
