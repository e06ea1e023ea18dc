"""Orthogonalized updates without a GPU: argument checks that come before the device, the layout of the structure, scratch sizes."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest

from tests.conftest import ROOT

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def abi():
    from paper_2609_27193_gb300 import build as B
    B.build()
    from paper_2609_27193_gb300 import _abi
    _abi.load()
    return _abi


def test_struct_layout_matches_c(abi):
    src = ('#include <stdio.h>\n#include <stddef.h>\n#include "layercheck.h"\nint main(void) {'
           + "".join('printf("%%zu ", offsetof(lc_mats, %s));' % f for f, _ in abi.lc_mats._fields_)
           + 'printf("%zu %d", sizeof(lc_mats), LC_ORTH_MAX_DIM); return 0; }')
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "l.c"), "w").write(src)
        subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), os.path.join(d, "l.c"), "-o", os.path.join(d, "l")],
                       check=True)
        got = [int(x) for x in subprocess.run([os.path.join(d, "l")], capture_output=True, text=True, check=True).stdout.split()]
    want = [getattr(abi.lc_mats, f).offset for f, _ in abi.lc_mats._fields_]
    assert got == want + [C.sizeof(abi.lc_mats), abi.LC_ORTH_MAX_DIM]


def test_refusals_before_the_device(abi):
    lib = abi.load()

    def mats(ptr=4096, stride=96, batch=96 * 64, dtype=abi.LC_BF16):
        return abi.lc_mats(ptr, stride, batch, dtype, 0)

    def says(word, u=None, b=1, m=64, n=96, mom=None, beta=0.9, steps=1, coef=(1.5, -0.5, 0.0), eps=1e-7, o=None, ws=8192, size=1 << 40):
        packed = (C.c_double * len(coef))(*coef) if coef else None
        st = lib.lc_orthogonalize(0, None, u or mats(), b, m, n, mom, beta, 1, steps, packed, eps, o or mats(1 << 20), ws, size)
        assert st != abi.LC_OK and word in lib.lc_last_error(), lib.lc_last_error()
    says(b"matrices of", m=0)
    says(b"matrices of", n=abi.LC_ORTH_MAX_DIM + 1)
    says(b"matrices of", b=-1)
    says(b"matrices of", b=65536)
    says(b"steps", steps=0)
    says(b"steps", steps=17)
    says(b"steps", coef=None)
    says(b"eps", eps=-1.0)
    says(b"eps", eps=float("nan"))
    says(b"beta", mom=mats(dtype=abi.LC_F32), beta=1.0)
    says(b"beta", mom=mats(dtype=abi.LC_F32), beta=float("nan"))
    says(b"fp32", mom=mats())
    says(b"bf16", o=mats(dtype=abi.LC_F32))
    says(b"unknown dtype", u=mats(dtype=9))
    says(b"element-aligned", u=mats(4097))
    says(b"strides", u=mats(stride=-1))
    says(b"strides", u=mats(stride=1 << 50))
    says(b"overlap", o=mats(stride=95))
    says(b"overlap", b=2, o=mats(batch=96 * 64 - 1))
    says(b"overlap", b=2, o=mats(batch=95, stride=96 * 2))
    says(b"grow", coef=(17.0, 0.0, 0.0))
    says(b"coefficients", coef=(float("inf"), 0.0, 0.0))
    says(b"workspace", m=640, size=16, n=96 * 8, u=mats(stride=768), o=mats(1 << 30, stride=768))
    says(b"256-byte", m=640, n=96 * 8, u=mats(stride=768), o=mats(1 << 30, stride=768), ws=8192 + 16)


def test_workspace(abi):
    """Room for X in fp32 and twice in fp16, and for A in fp32, A and B in fp16, padded to whole tiles; none for sizes that
    are refused."""
    size = abi.load().lc_orthogonalize_workspace
    for b, m, n in ((1, 1, 1), (5, 128, 4096), (1, 100, 20)):
        assert size(b, m, n) == size(b, n, m) == 0            # small ones stay in a cluster's memory
    for b, m, n in ((1, 129, 129), (1, 128, 4097), (1, 256, 256), (8, 1024, 256), (1, 4096, 14336), (3, 515, 1023)):
        lo, hi = sorted((m, n))
        assert size(b, m, n) >= b * 8 * (lo * hi + lo * lo)
        assert size(b, m, n) == size(b, n, m)
        assert size(b, m, n) < b * 8 * (lo + 256) * (hi + 256) * 2 + (152 << 18)
    for bad in ((0, 4, 4), (1, 0, 4), (1, 4, 0), (1, 4, abi.LC_ORTH_MAX_DIM + 1), (65536, 4, 4), (-1, 4, 4)):
        assert size(*bad) == 0


def test_without_a_device():
    from paper_2609_27193_gb300 import ops
    with pytest.raises(ValueError):
        ops.orthogonalize(torch.zeros(4, 4))
    for kw in (dict(steps=0), dict(steps=17), dict(coefficients=()), dict(coefficients=(1.0,)), dict(coefficients=[[1.0, 2.0]]),
               dict(steps=2, coefficients=((1.0, 2.0, 3.0), 4.0)), dict(steps=3, coefficients=((1.0, 2.0, 3.0),) * 2)):
        with pytest.raises(ValueError):
            ops.orthogonalize(torch.zeros(4, 4), **kw)
