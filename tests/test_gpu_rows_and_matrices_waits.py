"""The norm of a residual sum and orthogonalized updates when a wait inside a kernel runs out: a copy announces 16 bytes more
than it brings, every wait gives up after a second or so, what depends on it is NaN, and the next call is right."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import BF, F32, gen, randn  # noqa: E402
from tests.test_gpu_ops_waits import stalled  # noqa: E402, F401


@pytest.mark.parametrize("t,d,dt,rt", [(5000, 256, BF, BF), (5000, 1024, F32, F32), (1300, 4096, BF, F32), (320, 8192, BF, BF)])
def test_add_norm(stalled, t, d, dt, rt):  # noqa: F811
    """Sizes that go through the rings (other forms wait for nothing).  Every group's first row does not come; the rows that follow are not waited for."""
    from paper_2609_27193_gb300 import ops
    g = gen(t)
    x, r, w = randn(g, t, d, dtype=dt), randn(g, t, d, dtype=rt), 1 + randn(g, d, dtype=dt, spread=0.2)
    want = ops.add_norm(x, r, w, keep=True, out8=True)
    got = stalled(lambda: ops.add_norm(x, r, w, keep=True, out8=True))
    assert all(torch.isnan(v).all() for v in got[:3])
    assert all((v.e == 127).all() and (v.q == 0).all() for v in got[3:])
    again = ops.add_norm(x, r, w, keep=True, out8=True)
    assert all(torch.equal(p, q) for p, q in zip(again[:3], want[:3]))
    dy, ds = randn(g, t, d, dtype=dt), randn(g, t, d, dtype=rt)
    for total in (want[0], want[3]):
        want_g = ops.add_norm_grad(dy, ds, total, w, want[2])
        got = stalled(lambda: ops.add_norm_grad(dy, ds, total, w, want[2]))
        assert torch.isnan(got[0]).all() and torch.isnan(got[1]).all()
        assert all(torch.equal(p, q) for p, q in zip(ops.add_norm_grad(dy, ds, total, w, want[2]), want_g))


@pytest.mark.parametrize("shape", [(300, 500), (700, 150), (2, 129, 4200), (1100, 8000), (2048, 2048)])
def test_orthogonalize(stalled, shape):  # noqa: F811
    """Single tiles and pairs', whole products and splits of them; the momentum has moved all the same."""
    from paper_2609_27193_gb300 import ops
    g = gen(shape[-1])
    u, m0 = randn(g, *shape), randn(g, *shape)
    m = m0.clone()
    want = ops.orthogonalize(u, momentum=m)
    n = m0.clone()
    out = torch.zeros_like(want)
    stalled(lambda: ops.orthogonalize(u, momentum=n, out=out))
    assert torch.isnan(out).all() and torch.equal(n, m)
    ops.orthogonalize(u, momentum=m0, out=out)
    assert torch.equal(out, want)
