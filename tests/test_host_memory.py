"""The host calls that keep lists of their own return an error when there is no memory for them: nothing is thrown across
the C boundary (which would end the process).  In a child process whose address space is limited."""
import subprocess
import sys

import pytest

from paper_2502_13176_b200 import build as bkbuild

CHILD = """
import ctypes, resource, sys
import numpy as np
from ctypes import POINTER, c_double, c_int32, c_int64
from paper_2502_13176_b200 import binding as bk
lib = bk.lib()
n = 4096
sh = bk.make_shape(n, n, n, 128)
cap, off, imp = np.full(n * n, 16, np.int32), np.zeros(n * n, np.int64), np.ones(n * n)
info, stride = bk.PlanInfo(), c_int64(0)
params = bk.AllocParams(0.5, 1, 2, bk.SCOPE_MODEL, 16, 64, None, 0.0, 0, 1)
with open("/proc/self/statm") as f:
    used = int(f.read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (used + (32 << 20),) * 2)          # each list takes 64 MB and more
if sys.argv[1] == "plan":
    rc = lib.baklava_decode_plan(ctypes.byref(sh), cap.ctypes.data_as(POINTER(c_int32)), 1, 0, n, 64, 148, 0, 16 * n * n, None, 0,
                                 ctypes.byref(info))
else:
    rc = lib.baklava_allocate(ctypes.byref(sh), imp.ctypes.data_as(POINTER(c_double)), ctypes.byref(params), 16 * n * n,
                              cap.ctypes.data_as(POINTER(c_int32)), off.ctypes.data_as(POINTER(c_int64)), ctypes.byref(stride))
print("rc", rc)
"""


@pytest.mark.parametrize("call", ["plan", "allocate"])
def test_no_memory_is_an_error_code(call):
    bkbuild.build()
    run = subprocess.run([sys.executable, "-c", CHILD, call], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, (run.returncode, run.stderr[-500:])
    assert run.stdout.split()[-2:] == ["rc", "-4"]
