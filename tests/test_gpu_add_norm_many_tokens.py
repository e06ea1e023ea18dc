"""The gradient of the norm of a residual sum over rows whose offsets pass 32 bits, each different from the others: dweight
in whole numbers, where a row that is left out or counted twice shows, and dx of rows from all over."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_add_norm import ops  # noqa: E402, F401
from tests.test_gpu_ops import BF, F32, U, gen, norm_grad_ref, randn, values, within  # noqa: E402


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def whole(g, most, *shape, dtype):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("t,d,rt", [(300_000, 8192, BF), (290_001, 8191, BF), (300_000, 4096, F32), (600_011, 2051, F32)])
def test_gradient(ops, t, d, rt, kept):  # noqa: F811
    """dy of [-2, 2], sums of [-4, 4] and an rstd of 1/2, 1 or 2: a term of dweight is a multiple of 1/2 of at most 16, so all
    sums of up to 600,011 of them stay below 2^24 halves in practice (a hundredth of the worst, and asserted), exact in any
    order.  A checkpoint holds such sums exactly."""
    g = gen(t)
    dy, s, ds = whole(g, 2, t, d, dtype=BF), whole(g, 4, t, d, dtype=rt), whole(g, 3, t, d, dtype=rt)
    rstd = torch.exp2(whole(g, 1, t, dtype=F32))
    w = 1 + randn(g, d, dtype=BF, spread=0.1)
    assert t * d * s.element_size() > 1 << 31
    total = ops.act_save(s) if kept else s
    dx, dw = ops.add_norm_grad(dy, ds, total, w, rstd)
    ref = torch.zeros(d, dtype=torch.float64, device="cuda")
    most = torch.zeros_like(ref)
    for at in range(0, t, 10_000):
        terms = dy[at:at + 10_000].double() * s[at:at + 10_000].double() * rstd[at:at + 10_000, None].double()
        ref += terms.sum(0)
        most += terms.abs().sum(0)
    assert float(most.max()) < 2.0 ** 23
    assert torch.equal(dw.double(), ref)
    if kept:
        assert torch.equal(values(total.q[-64:], total.e[-64:])[:, :d], s[-64:].float())
    for at in (0, t // 3, t // 2 + 1, t - 64):
        rows = slice(at, at + 64)
        rdx, room, _, _, _, _ = norm_grad_ref(dy[rows], s[rows], w, None, rstd[rows])
        rdx = rdx + ds[rows].double()
        within(dx[rows], rdx, room + 4 * U * (rdx.abs() + ds[rows].double().abs()), "dx")
