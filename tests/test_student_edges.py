"""Calls of the student block's operators that need no GPU to go wrong: those without rows, the
sizes of workspaces, what the status read covers."""
import ctypes
import subprocess
import sys

import pytest

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


@pytest.mark.parametrize("rows,kind", [(0, 1), (0, 2), (1, 1), (64, 2)])
def test_a_norm_backward_of_no_rows_does_nothing(rows, kind):
    """In a process of its own: what goes wrong here takes the process with it."""
    code = """
import ctypes
from paper_2609_18145_gb300 import hcw as H
P = ctypes.c_void_p
before = H.hcw_launch_count()
rc = H.lib().hcw_residual_norm_bwd(None, None, None, None, None, %d, 1.0, %d, None, None, %d, None,
                                   1e-5, 0, 96, 1, P(1 << 20), None, None, None, None, None, None,
                                   None, 0, None)
assert rc == H.HCW_OK, rc
assert H.hcw_launch_count() == before
""" % (rows, kind, kind)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
