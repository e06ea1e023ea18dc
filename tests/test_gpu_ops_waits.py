"""The operators when a wait inside a kernel runs out: a copy announces 16 bytes more than it brings, every wait gives up
after a second, what depends on it is NaN, and the next call is right."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import BF, F32, gen, randn  # noqa: E402


@pytest.fixture()
def stalled():
    """Runs a call with the switch on; off again whatever happens."""
    from paper_2609_27193_gb300 import _abi
    lib = _abi.load()

    def run(call):
        _abi.check(lib.lc_ops_debug(_abi.LC_DEBUG_OPS_STALL))
        try:
            return call()
        finally:
            _abi.check(lib.lc_ops_debug(0))
            torch.cuda.synchronize()
    return run


@pytest.mark.parametrize("t,n,k,dt,gt", [(100, 70, 200, BF, F32), (2100, 300, 500, F32, F32), (2100, 300, 500, BF, BF),
                                         (300, 2560, 2816, BF, BF), (300, 2560, 2816, F32, F32)])
def test_weight_grad(stalled, dt, gt, t, n, k):
    """One tile, splits that are joined, and several tiles a pair.  The second CTA of a pair misses a copy; the first
    one's products read half of it."""
    from paper_2609_27193_gb300 import ops
    g = gen(t)
    dy, a = randn(g, t, n, dtype=dt), ops.act_save(randn(g, t, k, dtype=dt))
    want = ops.weight_grad(dy, a, dtype=gt)
    out = torch.zeros_like(want)
    stalled(lambda: ops.weight_grad(dy, a, grad=out))
    assert torch.isnan(out).all()
    ops.weight_grad(dy, a, grad=out)
    assert torch.equal(out, want)
    base = randn(g, n, k, dtype=gt)
    stalled(lambda: ops.weight_grad(dy, a, grad=base, accumulate=True))
    assert torch.isnan(base).all()


@pytest.mark.parametrize("t,d,dt,kind", [(5000, 256, BF, "rms"), (700, 1024, F32, "layer"), (400, 4096, BF, "layer"),
                                         (320, 16384, F32, "rms")])
def test_norm(stalled, kind, t, d, dt):
    """Every group's first row does not come; the rows that follow are not waited for."""
    from paper_2609_27193_gb300 import ops
    g = gen(t)
    x, dy, w = randn(g, t, d, dtype=dt), randn(g, t, d, dtype=dt), 1 + randn(g, d, dtype=dt, spread=0.2)
    b = randn(g, d, dtype=dt) if kind == "layer" else None
    want = ops.norm(x, w, b, kind=kind, keep=True)
    _, mean, rstd, act = want
    got = stalled(lambda: ops.norm(x, w, b, kind=kind, keep=True))
    assert torch.isnan(got[0]).all() and torch.isnan(got[2]).all() and (mean is None or torch.isnan(got[1]).all())
    assert (got[3].e == 127).all() and (got[3].q == 0).all()
    again = ops.norm(x, w, b, kind=kind, keep=True)
    assert all(p is q is None or torch.equal(p, q) for p, q in zip(again[:3], want[:3]))
    assert torch.equal(again[3].q, act.q) and torch.equal(again[3].e, act.e)
    for seen in (x, act):
        for bias in (True, False):
            right = ops.norm_grad(dy, seen, w, mean, rstd, bias=bias)
            lost = stalled(lambda: ops.norm_grad(dy, seen, w, mean, rstd, bias=bias))
            assert all(p is None or torch.isnan(p).all() for p in lost)
            assert all(p is q is None or torch.equal(p, q) for p, q in zip(ops.norm_grad(dy, seen, w, mean, rstd, bias=bias), right))
