"""What the operators' binding refuses before anything runs on the GPU."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import BF, gen, randn  # noqa: E402


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import ops
    return ops


def test_a_checkpoint_that_changed_after_it_was_made(ops):
    g = gen(61)
    t, d = 40, 300
    x, dy, w = randn(g, t, d, dtype=BF), randn(g, t, d, dtype=BF), torch.ones(d, dtype=BF, device="cuda")
    good = ops.act_save(x)
    _, mean, rstd = ops.norm(x, w)
    want = ops.act_load(good)

    def broken():
        for field, value in (("q", good.q[:, :256]), ("q", good.q[:t - 1]), ("q", good.q.view(torch.uint8)), ("q", good.q.view(-1)),
                             ("q", good.q.t().contiguous().t()), ("e", good.e[:, :2]), ("e", good.e[:t - 1]), ("e", good.e.float()),
                             ("e", good.e.t().contiguous().t()), ("dim", 10 ** 6), ("dim", 0), ("dim", -5), ("e", good.e.cpu())):
            a = ops.Act(good.q, good.e, d)
            setattr(a, field, value)
            yield a
    for a in broken():
        with pytest.raises(ValueError):
            ops.act_load(a)
        with pytest.raises(ValueError):
            ops.act_save(x, a)
        with pytest.raises(ValueError):
            ops.norm(x, w, keep=a)
        with pytest.raises(ValueError):
            ops.norm_grad(dy, a, w, mean, rstd)
        with pytest.raises(ValueError):
            ops.weight_grad(dy, a)
    a = ops.Act(good.q, good.e, d)
    a.e = None
    with pytest.raises(ValueError):
        ops.weight_grad(dy, a)
    assert torch.equal(ops.act_load(good), want)


def test_one_row_may_have_any_stride(ops):
    g = gen(62)
    x, dy = randn(g, 1, 200, dtype=BF), randn(g, 1, 70, dtype=BF)
    want = ops.act_save(x)
    a = ops.Act(torch.zeros(256, 1, dtype=torch.int8, device="cuda").t(), torch.zeros(2, 1, dtype=torch.int8, device="cuda").t(), 200)
    assert a.q.stride() == (1, 1) and a.e.stride() == (1, 1)
    ops.act_save(x, a)
    assert torch.equal(a.q, want.q) and torch.equal(a.e, want.e) and torch.equal(ops.act_load(a), ops.act_load(want))
    assert torch.equal(ops.weight_grad(dy, a), ops.weight_grad(dy, want))


def test_inputs_that_autograd_would_lose(ops):
    """A parameter that goes through a forward call would come out detached: refused while grad mode is on."""
    g = gen(63)
    t, d = 12, 64
    x, ids = randn(g, t, d), torch.randint(0, t, (t,), generator=g, device="cuda")
    w, b = torch.nn.Parameter(torch.ones(d, device="cuda")), torch.nn.Parameter(torch.zeros(d, device="cuda"))
    table = torch.nn.Parameter(x.clone())
    for call in (lambda: ops.embed(table, ids), lambda: ops.norm(table, w.detach()), lambda: ops.norm(x, w),
                 lambda: ops.norm(x, w.detach(), b), lambda: ops.norm(x, w.detach(), out=table)):
        with pytest.raises(RuntimeError, match="autograd"):
            call()
        with torch.no_grad():
            call()
    # where torch differentiates by itself, and where nothing requires a gradient
    with torch.inference_mode():
        ops.norm(x, w, out=torch.empty_like(x))
    y, mean, rstd = ops.norm(x, w.detach())
    ops.norm_grad(y, x, w, mean, rstd)

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            y, mean, rstd = ops.norm(x, w)
            ctx.save_for_backward(x, w, mean, rstd)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w, mean, rstd = ctx.saved_tensors
            dx, dw, _ = ops.norm_grad(dy.contiguous(), x, w, mean, rstd)
            return dx, dw
    p = x.clone().requires_grad_()
    Norm.apply(p, w).square().sum().backward()
    q, v = x.double().requires_grad_(), w.detach().double().requires_grad_()
    torch.nn.functional.layer_norm(q, (d,), v, None, 1e-5).square().sum().backward()
    # two fp32 norms of 64 columns and sums of 12 rows: far below this
    assert (p.grad - q.grad).abs().max() < 1e-4 and (w.grad - v.grad).abs().max() < 1e-4


def test_what_is_written_counts_as_written(ops):
    """torch refuses a backward pass over saved tensors that a call has overwritten."""
    g = gen(64)
    t, d = 12, 128
    x, dy, w = randn(g, t, d), randn(g, t, d), torch.ones(d, device="cuda")
    ids = torch.randint(0, t, (t,), generator=g, device="cuda")
    a = ops.act_save(x)
    _, mean, rstd = ops.norm(x, w)

    def fresh(*shape):
        return torch.zeros(*shape, device="cuda")
    o, p, q = fresh(t, d), fresh(d), fresh(d)
    b = ops.act_save(x)
    for tensors, call in (((o,), lambda: ops.embed(x, ids, out=o)), ((o,), lambda: ops.embed_grad(dy, ids, grad=o)),
                          ((b.q, b.e), lambda: ops.act_save(x, b)), ((o,), lambda: ops.act_load(a, out=o)),
                          ((o, b.q, b.e), lambda: ops.norm(x, w, out=o, keep=b)),
                          ((o, p, q), lambda: ops.norm_grad(dy, x, w, mean, rstd, dx=o, dweight=p, dbias=q))):
        before = [v._version for v in tensors]
        call()
        assert all(v._version > n for v, n in zip(tensors, before))
    dw = fresh(d, d)
    n = dw._version
    ops.weight_grad(dy, a, grad=dw)
    assert dw._version > n
    s = torch.ones(t, d, device="cuda", requires_grad=True)
    y = s * o
    with torch.no_grad():
        ops.norm(x, w, out=o)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_an_output_that_does_not_fit(ops):
    """16 TB: what a program catches around torch's own allocations it catches here."""
    dy, ids = torch.zeros(1, 4096, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):
        ops.embed_grad(dy, ids, 10 ** 9)


def test_a_gradient_of_another_vocabulary(ops):
    dy, ids = torch.ones(3, 16, device="cuda"), torch.tensor([0, 11, 19], device="cuda")
    grad = torch.zeros(20, 16, device="cuda")
    with pytest.raises(ValueError, match="vocab"):
        ops.embed_grad(dy, ids, 10, grad=grad)
    assert (grad == 0).all()
    ops.embed_grad(dy, ids, 20, grad=grad)
    assert (grad[ids] == 1).all() and float(grad.sum()) == 48
