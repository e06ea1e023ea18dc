"""Updates whose squares lie below fp32's range: their norm is as good as any other's, with eps = 0 too, in the one-cluster
form and in the products' (a CTA's tiles and a pair's), against the definition in 64 bits as in test_gpu_orthogonalize.py."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import BF, F32, gen, randn  # noqa: E402
from tests.test_gpu_orthogonalize import check, definition  # noqa: E402

SHAPES = [(70, 90), (90, 70), (128, 700), (300, 500), (1100, 1200), (1200, 1100)]


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import ops
    return ops


def small(g, scale, *shape, dtype=F32):
    """Rounded once to the type (below 1.2e-38 to a multiple of 2^-149)."""
    u = randn(g, *shape).double()
    return (u / u.abs().max() * scale).to(dtype)


@pytest.mark.parametrize("scale", [1e-10, 1e-12, 1e-13, 1e-18, 1e-20, 1e-21, 1e-23, 1e-30, 1e-38, 1e-42])
@pytest.mark.parametrize("m,n", SHAPES)
def test_magnitudes(ops, m, n, scale):
    u = small(gen(m), scale, m, n)
    check(lambda k: ops.orthogonalize(u, steps=k, eps=0.0), u, eps=0.0)
    # an eps of the norm's size
    eps = float(u.double().norm()) / 3
    check(lambda k: ops.orthogonalize(u, steps=k, eps=eps), u, eps=eps)


@pytest.mark.parametrize("m,n", SHAPES)
def test_sixteen_bits_and_momentum(ops, m, n):
    g = gen(m + n)
    u = small(g, 1e-25, 2, m, n, dtype=BF)
    m0 = small(g, 1e-24, 2, m, n)
    beta = 0.5                                    # powers of two: the momentum and the update are exact to 2^-23 of what goes in
    got = {k: ops.orthogonalize(u, momentum=m0.clone(), beta=beta, steps=k, eps=0.0) for k in (2, 5)}
    after = m0.double() + (1 - beta) * (u.double() - m0.double())
    up = u.double() + beta * (after - u.double())
    for b in range(2):
        check(lambda k: got[k][b], up[b], eps=0.0)


@pytest.mark.parametrize("m,n", [(70, 90), (300, 500)])
def test_a_batch_of_all_magnitudes(ops, m, n):
    """Each matrix by its own norm; a matrix of zeros among them."""
    scales = [1e30, 1e20, 1.0, 1e-11, 1e-13, 1e-22, 1e-40, 0.0]
    u = torch.stack([small(gen(k), s, m, n) for k, s in enumerate(scales)])
    got = {k: ops.orthogonalize(u, steps=k, eps=0.0) for k in (2, 5)}
    for b, s in enumerate(scales):
        if s:
            check(lambda k: got[k][b], u[b], eps=0.0)
        else:
            assert torch.isnan(got[5][b]).all()


@pytest.mark.parametrize("m,n", [(64, 80), (300, 500)])
def test_few_values(ops, m, n):
    """One value of a size of its own over others that add nothing to the norm, and one that is all there is."""
    for top, rest in ((1e-13, 1e-30), (1e-20, 1e-40), (1e-41, 0.0), (2.0 ** -149, 0.0), (2.0 ** -40, 1e-20), (2.0 ** -41, 1e-20)):
        u = small(gen(3), rest, m, n)
        u[m // 2, n - 1] = top
        got = ops.orthogonalize(u, eps=0.0).double()
        ref = definition(u, eps=0.0)
        assert abs(float(got[m // 2, n - 1] - ref[m // 2, n - 1])) <= 2.0 ** -8
        got[m // 2, n - 1] = ref[m // 2, n - 1] = 0
        assert (got.abs() <= 1.02 * ref.abs() + 1e-8).all()


@pytest.mark.parametrize("m,n", [(64, 80), (300, 500), (1100, 1200)])
@pytest.mark.parametrize("eps", [1e-7, 1e-30, 1e-42, 1e-300])
def test_zeros(ops, m, n, eps):
    """Zeros stay zeros with any eps that is not 0."""
    u = torch.zeros(m, n, device="cuda")
    assert (ops.orthogonalize(u, eps=eps) == 0).all()
    assert torch.isnan(ops.orthogonalize(u, eps=0.0)).all()
