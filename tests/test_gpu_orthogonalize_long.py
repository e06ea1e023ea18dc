"""Orthogonalized updates up to the longest side that there may be: matrices of which few columns (or rows) are not zero,
which come out as the matrix of those columns alone, with zeros between; and a large matrix with one value a row."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import BF, F32, gen, randn  # noqa: E402
from tests.test_gpu_orthogonalize import NEAR, check, definition  # noqa: E402


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import ops
    return ops


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("m", [1, 100, 130, 300, 1100])
def test_longest_side(ops, m, turned, dtype):
    from paper_2609_27193_gb300._abi import LC_ORTH_MAX_DIM as n
    g = gen(m)
    # one column of every 64, and some more, the first and the last among them
    at = torch.arange(0, n, 64, device="cuda") + torch.randint(0, 64, (n // 64,), generator=g, device="cuda")
    more = torch.randint(0, n, (400,), generator=g, device="cuda")
    at = torch.unique(torch.cat([at, more, torch.tensor([0, n - 1], device="cuda")]))
    few = randn(g, m, len(at), dtype=dtype, spread=1e-3)
    u = torch.zeros(m, n, dtype=dtype, device="cuda")
    u[:, at] = few
    u = u.t().contiguous() if turned else u
    got = {k: ops.orthogonalize(u, steps=k) for k in (2, 5)}
    got = {k: v.t() if turned else v for k, v in got.items()}
    check(lambda k: got[k][:, at], few)
    zero = torch.ones(n, dtype=torch.bool, device="cuda")
    zero[at] = False
    assert (got[5][:, zero] == 0).all()


def test_one_value_a_row(ops):
    """Every singular value is 1 / sqrt(m): the polynomial of it at each place, zeros elsewhere; arrays beyond 2^32 bytes."""
    m, n = 24000, 65536
    g = gen(7)
    at = torch.randperm(n, generator=g, device="cuda")[:m]
    rows = torch.arange(m, device="cuda")
    sign = torch.randint(0, 2, (m,), generator=g, device="cuda").float() * 2 - 1
    u = torch.zeros(m, n, device="cuda")
    u[rows, at] = sign
    got = ops.orthogonalize(u)
    # (a diagonal matrix of m such values in place of the rows)
    want = float(definition(torch.eye(1, device="cuda") / math.sqrt(m), 5, eps=1.0 - 1.0 / math.sqrt(m)))
    seen = got[rows, at].double() * sign.double()
    assert ((seen - want).abs() <= NEAR * want).all()
    got[rows, at] = 0
    assert (got == 0).all()
