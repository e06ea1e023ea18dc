"""Calls with nothing to do, up to where the device is looked for: without a GPU they end with a status as any other call's.
In a process of their own, which a division by zero would end (on the processors that trap on one)."""
import signal
import subprocess
import sys

import pytest

from tests.conftest import ROOT

CALLS = """
import ctypes as C
from paper_2609_27193_gb300 import build as B
B.build()
from paper_2609_27193_gb300 import _abi
lib = _abi.load()
F, H = _abi.LC_F32, _abi.LC_BF16
none = -1                      # a device that there is not
def rows(at, d): return _abi.lc_rows(at << 20, d, H, 0)
def mats(at, m, n, dtype): return _abi.lc_mats(at << 20, n, m * n, dtype, 0)
act = _abi.lc_act(9 << 20, 384, 10 << 20, 3)
one = (C.c_double * 3)(1.5, -0.5, 0.0)
for m, n in ((1, 1), (64, 96), (300, 500), (1100, 1200), (9000, 130), (65536, 65536)):
    assert lib.lc_orthogonalize_workspace(0, m, n) == 0
    for momentum in (None, mats(2, m, n, F)):
        st = lib.lc_orthogonalize(none, None, mats(1, m, n, H), 0, m, n, momentum, 0.9, 1, 1, one, 1e-7, mats(3, m, n, H), None, 0)
        assert st == _abi.LC_ERR_INVALID_ARG and b"device -1" in lib.lc_last_error(), lib.lc_last_error()
for d in (1, 300):
    for st in (lib.lc_add_norm(none, None, rows(1, d), rows(2, d), 0, d, 3 << 20, F, 1e-5, rows(4, d), rows(5, d), 6 << 20, act, None),
               lib.lc_add_norm_grad(none, None, rows(1, d), rows(2, d), rows(3, d), None, 0, d, 4 << 20, F, 5 << 20, rows(6, d), 7 << 20, F, 0,
                                    8 << 20, lib.lc_norm_grad_workspace(0, d)),
               lib.lc_norm(none, None, _abi.LC_NORM_RMS, rows(1, d), 0, d, 3 << 20, None, F, 1e-5, rows(5, d), None, 6 << 20, None),
               lib.lc_weight_grad(none, None, rows(1, d), act, 0, d, d, rows(2, d), 0, None, 0),
               lib.lc_act_save(none, None, rows(1, d), 0, d, act)):
        assert st == _abi.LC_ERR_INVALID_ARG and b"device -1" in lib.lc_last_error(), lib.lc_last_error()
print("done")
"""


def test_no_rows_and_no_matrices():
    pytest.importorskip("torch")
    r = subprocess.run([sys.executable, "-c", CALLS], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode != -signal.SIGFPE, "a division by zero"
    assert r.returncode == 0 and r.stdout.strip() == "done", r.stderr[-2000:]
