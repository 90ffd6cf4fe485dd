"""CPU-only checks of what the products with 4-bit weights need, by the limits that include/stom_w4.h gives."""
import ctypes as C

import pytest
import torch

from test_kv_cpu import P, oqm  # noqa: F401


def need(oqm, rows, n, k, group):  # noqa: F811
    desc = oqm.W4Desc(codes=P, scale=P, zero=None, n=n, k=k, group=group, meta_dtype=0, code_stride=-(-k // 32) * 16,
                      meta_stride=k // group)
    return oqm.lib().stom_w4_workspace_bytes(C.byref(desc), rows)


@pytest.mark.parametrize("rows,k,group", [(8, 3840, 32), (5, 5632, 32), (1, 17408, 32), (8, 4096, 128), (5, 6400, 128),
                                          (1, 27648, 128), (8, 4096, 64)])
def test_few_tokens_need_no_workspace_up_to_the_limits_that_are_given(oqm, rows, k, group):  # noqa: F811
    assert need(oqm, rows, 4608, k, group) == 0
    assert need(oqm, rows, 4608, k + group, group) > 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="asks without a device")
@pytest.mark.parametrize("n", [16, 1184, 1185, 4608, 28416, 28417, 151001])
def test_without_a_device_nothing_is_taken_for_granted_of_its_size(oqm, n):  # noqa: F811
    """9 to 16 tokens need a workspace or not by the device's number of multiprocessors."""
    assert need(oqm, 8, n, 512, 64) == 0 and need(oqm, 9, n, 512, 64) > 0 and need(oqm, 16, n, 512, 64) > 0
