"""The wait that the kernels' barriers are waited on with ends by itself, and soon after it has been called off.  (A kernel in
which it runs out sets STOM_FLAG_TIMEOUT; that no call does is asserted wherever flags are read.)"""
import ctypes as C
import subprocess
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu


def test_a_wait_ends_at_its_limit_and_when_it_is_called_off(tmp_path):
    from paper_2510_18269_b200 import build
    lib = tmp_path / "waits.so"
    src = Path(__file__).with_name("bounded_wait.cu")
    r = subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-shared", str(src), "-o", str(lib)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = (C.c_ulonglong * 8)()
    ms = 1000000
    assert C.CDLL(str(lib)).run_waits(C.c_ulonglong(20 * ms), C.c_ulonglong(3 * ms), out) == 0
    limit, off, gone, arrived = [(out[2 * i], out[2 * i + 1]) for i in range(4)]
    assert limit[0] == 0 and 20 * ms <= limit[1] < 22 * ms
    assert off[0] == 0 and off[1] < ms // 2
    assert gone[0] == 0 and gone[1] < ms // 10
    assert arrived[0] == 1 and arrived[1] < ms // 10
