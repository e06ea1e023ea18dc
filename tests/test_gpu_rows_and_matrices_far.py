"""The norm of a residual sum and orthogonalized updates where offsets pass 32 bits: many rows, many matrices, rows far apart;
the largest batch and the longest matrix of the one-cluster form."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import BF, F32, gen, randn  # noqa: E402
from tests.test_gpu_orthogonalize import check  # noqa: E402


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t,d", [(300_000, 8192), (290_001, 8191)])
def test_add_norm(t, d):
    """Rows of x and of the stream repeat; the last rows' results are the first ones'."""
    from paper_2609_27193_gb300 import ops
    g = gen(1)
    x, r, w = randn(g, 1, d, dtype=BF), randn(g, 1, d, dtype=BF), 1 + randn(g, d, dtype=BF, spread=0.1)
    s, y, rstd, kept, y8 = ops.add_norm(x.expand(t, d), r.expand(t, d), w, keep=True, out8=True)
    for v in (s, y, kept.q, y8.q):
        assert torch.equal(v[-1], v[0]) and torch.equal(v[t // 2], v[0])
    want = ops.add_norm(x.expand(400, d), r.expand(400, d), w)
    assert torch.equal(y[-1], want[1][0]) and torch.equal(s[-1], want[0][0])
    del y, y8
    dy = randn(g, 1, d, dtype=BF).expand(t, d)
    dx, _ = ops.add_norm_grad(dy, s, kept, w, rstd)
    assert torch.equal(dx[-1], dx[0]) and torch.equal(dx[t // 2], dx[0])
    del dx
    dx, _ = ops.add_norm_grad(dy, s, s, w, rstd, dx=s[:1].expand(t, d).clone())
    assert torch.equal(dx[-1], dx[0])


@pytest.mark.parametrize("b,m,n", [(2100, 1024, 1024), (17000, 256, 512), (65535, 60, 70)])
def test_many_matrices(b, m, n):
    from paper_2609_27193_gb300 import ops
    u = randn(gen(b), 1, m, n)
    got = {k: ops.orthogonalize(u.expand(b, m, n), steps=k) for k in (2, 5)}
    for v in got.values():
        assert torch.equal(v[-1], v[0]) and torch.equal(v[b // 2], v[0])
    check(lambda k: got[k][-1], u[0])


@pytest.mark.parametrize("m,n", [(1030, 1100), (1100, 1030), (100, 700)])
def test_rows_far_apart(m, n):
    from paper_2609_27193_gb300 import ops
    far = (1 << 33) // m // 64 * 64 + 64
    buf = torch.empty(m * far, dtype=BF, device="cuda")
    v = buf.view(m, far)
    u, o = v[:, :n], v[:, 4096:4096 + n]
    u.copy_(randn(gen(m), m, n))
    check(lambda k: ops.orthogonalize(u, steps=k), u)
    want = ops.orthogonalize(u.contiguous())
    # columns of one buffer lie across one another: refused as an output
    from paper_2609_27193_gb300._abi import LCError
    with pytest.raises(LCError):
        ops.orthogonalize(u, out=o)
    ops.orthogonalize(u.contiguous(), out=o)
    assert (o.double() - want.double()).norm() < 1e-2 * want.double().norm()


def test_longest_matrices_of_a_cluster():
    from paper_2609_27193_gb300 import ops
    for m, n in ((128, 4096), (128, 4097), (129, 4096), (4095, 127), (1, 4096), (1, 5000), (5000, 1)):
        u = randn(gen(n), m, n)
        check(lambda k: ops.orthogonalize(u, steps=k), u)
