"""Orthogonalized updates of up to 128 rows or columns when a wait runs out: nobody hears of the first product, every thread
gives up after a second, nothing more is issued, the output is NaN, and the next call is right."""
import time

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import gen, randn  # noqa: E402
from tests.test_gpu_ops_waits import stalled  # noqa: E402, F401


@pytest.mark.parametrize("shape", [(1, 1), (60, 70), (3, 50, 40), (100, 700), (700, 100), (128, 4096)])
def test_one_cluster(stalled, shape):  # noqa: F811
    """One CTA, several, sixteen; the momentum has moved all the same."""
    from paper_2609_27193_gb300 import ops
    g = gen(shape[-1])
    u, m0 = randn(g, *shape), randn(g, *shape)
    m = m0.clone()
    want = ops.orthogonalize(u, momentum=m)
    n = m0.clone()
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    start = time.monotonic()
    stalled(lambda: ops.orthogonalize(u, momentum=n, out=out))
    took = time.monotonic() - start
    assert torch.isnan(out).all() and torch.equal(n, m)
    # one wait of a second for all fifteen products, and a tenth of one before the memory is given back
    assert 0.5 < took < 3.0
    ops.orthogonalize(u, momentum=m0, out=out)
    assert torch.equal(out, want)
