"""The operators of a training step without a GPU: argument checks that come
before the device, the layout of their structures, scratch sizes."""
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
    structs = {"lc_rows": abi.lc_rows, "lc_act": abi.lc_act}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "layercheck.h"', "int main(void) {"]
    for name, cls in structs.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in cls._fields_]
    for c in ("LC_I32", "LC_I64", "LC_NORM_LAYER", "LC_NORM_RMS", "LC_NORM_MAX_DIM", "LC_ACT_BLOCK"):
        lines.append('printf("%s %%d\\n", %s);' % (c, c))
    lines.append("return 0; }")
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "layout.c"), os.path.join(d, "layout")
        open(src, "w").write("\n".join(lines))
        subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), src, "-o", exe], check=True)
        got = dict(l.split() for l in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines())
    for name, value in got.items():
        if "." in name:
            cls, field = name.split(".")
            assert int(value) == getattr(structs[cls], field).offset, name
        elif name in structs:
            assert int(value) == C.sizeof(structs[name]), name
        else:
            assert int(value) == getattr(abi, name), name


def rows(abi, ptr=4096, stride=64, dtype=None):
    return abi.lc_rows(ptr, stride, abi.LC_BF16 if dtype is None else dtype, 0)


def test_refusals_before_the_device(abi):
    lib = abi.load()
    bad = abi.LC_ERR_INVALID_ARG
    r, w = rows(abi), rows(abi, 8192)
    act = abi.lc_act(4096, 128, 8192, 1)

    def says(word, status):
        assert status == bad and word in lib.lc_last_error(), lib.lc_last_error()
    says(b"rows of", lib.lc_embed(0, None, r, 0, 64, 64, abi.LC_I64, 8, 1.0, w))
    says(b"tokens", lib.lc_embed(0, None, r, 8, 64, 64, abi.LC_I64, -1, 1.0, w))
    says(b"id type", lib.lc_embed(0, None, r, 8, 64, 64, 7, 8, 1.0, w))
    says(b"table is NULL", lib.lc_embed(0, None, None, 8, 64, 64, abi.LC_I64, 8, 1.0, w))
    says(b"unknown dtype", lib.lc_embed(0, None, rows(abi, dtype=9), 8, 64, 64, abi.LC_I64, 8, 1.0, w))
    says(b"element-aligned", lib.lc_embed(0, None, rows(abi, 4097), 8, 64, 64, abi.LC_I64, 8, 1.0, w))
    says(b"ids is not", lib.lc_embed(0, None, r, 8, 64, 68, abi.LC_I64, 8, 1.0, w))
    says(b"stride", lib.lc_embed(0, None, r, 8, 64, 64, abi.LC_I64, 8, 1.0, rows(abi, 8192, 63)))
    says(b"stride", lib.lc_embed(0, None, rows(abi, stride=-64), 8, 64, 64, abi.LC_I64, 8, 1.0, w))
    says(b"another type", lib.lc_embed(0, None, r, 8, 64, 64, abi.LC_I64, 8, 1.0, rows(abi, 8192, 64, abi.LC_F32)))
    says(b"kind", lib.lc_norm(0, None, 5, r, 8, 64, 64, None, abi.LC_BF16, 1e-5, w, 64, 64, None))
    says(b"mean goes with", lib.lc_norm(0, None, abi.LC_NORM_RMS, r, 8, 64, 64, None, abi.LC_BF16, 1e-5, w, 64, 64, None))
    says(b"mean goes with", lib.lc_norm(0, None, abi.LC_NORM_LAYER, r, 8, 64, 64, None, abi.LC_BF16, 1e-5, w, None, 64, None))
    says(b"eps", lib.lc_norm(0, None, abi.LC_NORM_LAYER, r, 8, 64, 64, None, abi.LC_BF16, float("nan"), w, 64, 64, None))
    says(b"weight", lib.lc_norm(0, None, abi.LC_NORM_LAYER, r, 8, 64, None, None, abi.LC_BF16, 1e-5, w, 64, 64, None))
    grad = lambda x, kept: lib.lc_norm_grad(0, None, abi.LC_NORM_RMS, r, x, kept, 8, 64, 64, abi.LC_BF16, None, 64,  # noqa: E731
                                            w, None, None, abi.LC_F32, 0, None, 0)
    says(b"one of x", grad(None, None))
    says(b"one of x", grad(r, act))
    for broken in (abi.lc_act(4104, 128, 8192, 1), abi.lc_act(4096, 120, 8192, 1), abi.lc_act(4096, 112, 8192, 1),
                   abi.lc_act(4096, 128, 8192, 0)):
        says(b"checkpoint", lib.lc_act_save(0, None, r, 8, 64, broken))
        says(b"checkpoint", lib.lc_weight_grad(0, None, r, broken, 8, 64, 64, w, 0, None, 0))
    says(b"checkpoint is NULL", lib.lc_act_load(0, None, None, 8, 64, w))
    says(b"rows of", lib.lc_weight_grad(0, None, r, act, 8, 0, 64, w, 0, None, 0))
    if not torch.cuda.is_available():
        says(b"device 0", lib.lc_act_save(0, None, r, 8, 64, act))
    says(b"device 99", lib.lc_act_save(99, None, r, 8, 64, act))


def test_workspace_sizes(abi):
    lib = abi.load()
    assert lib.lc_embed_grad_workspace(0, 100, 64) == 0
    assert lib.lc_embed_grad_workspace(-5, 100, 64) == 0
    assert lib.lc_norm_grad_workspace(0, 64) == 0
    sizes = [lib.lc_embed_grad_workspace(n, 1000, 512) for n in (1, 100, 10000, 1000000)]
    assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[1] > 0      # few tokens need none
    # two lists of ids and positions, and parts that stay far below the gradient's own traffic
    assert sizes[-1] < 16 * 1000000 + 64 * 1024 * 1024
    assert lib.lc_norm_grad_workspace(10 ** 9, 4096) == lib.lc_norm_grad_workspace(10 ** 6, 4096)
    assert lib.lc_norm_grad_workspace(7, 4096) == 7 * 2 * 4096 * 4


def test_act_checks_its_tensors(abi):
    from paper_2609_27193_gb300 import ops
    q, e = torch.zeros(4, 256, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.int8)
    a = ops.Act(q, e, 200)
    assert a.rows == 4 and a.nbytes == 4 * 258
    for bad in ((q.float(), e, 200), (q, e, 257), (q[:, :200], e, 200), (q, e[:, :1], 200), (q[:3], e, 200),
                (q.t().contiguous().t(), e, 200), (q, e, 0)):
        with pytest.raises(ValueError):
            ops.Act(*bad)
    with pytest.raises(ValueError):
        ops.act_save(torch.zeros(2, 4))
