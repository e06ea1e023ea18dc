"""The norm of a residual sum and its gradient, against their definitions in 64 bits, with the bounds of
test_gpu_ops.py: a sum over a row is off by at most SUMS roundings of the sum of its terms' magnitudes, a sum over t
tokens by t + 16 of them."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import BF, F32, SUMS, U, gen, norm_grad_ref, quantize, randn, strided, values, within  # noqa: E402

TYPES = [(BF, BF), (BF, F32), (F32, F32)]
# the forms: a warp or several a row, through rings or not, widths off 4 and off 128, the widest
SHAPES = [(1, 1), (1, 256), (3, 5), (4, 9000), (8, 300), (9, 300), (16, 250), (17, 250), (64, 256), (5, 127), (6, 129), (17, 520), (9, 915), (33, 1024), (300, 768), (4, 4100),
          (7, 8191), (2, 12296), (3, 16384), (4200, 96), (5000, 256), (700, 1000), (613, 2048), (620, 4096), (305, 8192), (310, 16384), (2500, 2052)]


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import ops
    return ops


def check_forward(x, r, w, s, y, rstd, keep, y8, eps=1e-5):
    d = x.shape[1]
    total = x.double() + r.double()
    within(s, total, U * total.abs(), "sum")
    ref = 1 / (total.square().mean(1) + eps).sqrt()
    within(rstd, ref, (SUMS + 6) * U * ref, "rstd")
    yref = total * ref[:, None] * w.double()
    room = (SUMS + 10) * U * yref.abs()
    if y is not None:
        within(y, yref, room, "y")
    if keep is not None:
        q, e, _ = quantize(x.float() + r.float())
        assert torch.equal(keep.q, q) and torch.equal(keep.e, e)
    if y8 is not None:
        got, step = values(y8.q, y8.e), torch.exp2(y8.e.double()).repeat_interleave(128, 1)[:, :d]
        assert (got[:, d:] == 0).all()
        off = (got[:, :d].double() - yref).abs()
        assert (off <= step / 2 + room).all()
        most = torch.zeros_like(y8.e, dtype=torch.float64)
        for b in range(most.shape[1]):
            most[:, b] = yref[:, b * 128:(b + 1) * 128].abs().amax(1)
        one = torch.exp2(y8.e.double())
        near = 1 + (SUMS + 10) * U
        assert (127 * one * near >= most).all() and ((63.5 * one <= most * near) | (y8.e == -126)).all()


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("t,d", SHAPES)
def test_add_norm(ops, t, d, dt, rt):
    g = gen(t * d)
    src, rsrc = randn(g, t, d, dtype=dt, spread=0.5), randn(g, t, d, dtype=rt)
    for lead, extra, wt in ((0, 0, dt), (8, 16, F32), (1, 3, BF)):
        w = 1 + randn(g, d, dtype=wt, spread=0.2)
        x, _ = strided(src, lead, extra)
        r, _ = strided(rsrc, lead, extra)
        out, buf = strided(torch.zeros(t, d, dtype=dt, device="cuda"), lead, extra)
        total, sbuf = strided(torch.zeros(t, d, dtype=rt, device="cuda"), lead, extra)
        s, y, rstd, keep, y8 = ops.add_norm(x, r, w, out=out, sum=total, keep=True, out8=True)
        assert s.data_ptr() == total.data_ptr() and y.data_ptr() == out.data_ptr()
        check_forward(x, r, w, s, y, rstd, keep, y8)
        # each output alone gives the same bits
        s2, y2, rstd2 = ops.add_norm(x, r, w)
        assert torch.equal(s2, s) and torch.equal(y2, y) and torch.equal(rstd2, rstd)
        s3, none, rstd3, only = ops.add_norm(x, r, w, out=False, out8=True)
        assert none is None and torch.equal(s3, s) and torch.equal(only.q, y8.q) and torch.equal(only.e, y8.e)
        # in place, into a checkpoint that is there
        again = ops.Act.empty(t, d, "cuda")
        r2, _ = strided(rsrc, lead, extra)
        s4, y4, rstd4 = ops.add_norm(x, r2, w, sum=r2, keep=again)
        assert s4.data_ptr() == r2.data_ptr() and torch.equal(r2, s) and torch.equal(y4, y) and torch.equal(again.q, keep.q)
        out.fill_(77.0)
        total.fill_(77.0)
        assert (buf == 77.0).all() and (sbuf == 77.0).all()


def test_values_that_are_not_finite(ops):
    for t, d in ((40, 256), (700, 2048)):
        g = gen(d)
        x, r, w = randn(g, t, d, dtype=BF), randn(g, t, d, dtype=BF), randn(g, d, dtype=BF)
        want = ops.add_norm(x, r, w, keep=True, out8=True)
        x[3, 200], r[5, 130], x[7, 0], r[7, 0] = math.nan, math.inf, math.inf, -math.inf
        s, y, rstd, keep, y8 = ops.add_norm(x, r, w, keep=True, out8=True)
        bad = [3, 5, 7]
        ok = torch.ones(t, dtype=torch.bool)
        ok[bad] = False
        assert torch.equal(s[ok], want[0][ok]) and torch.equal(y[ok], want[1][ok]) and torch.equal(y8.q[ok], want[4].q[ok])
        assert torch.isnan(s[3, 200]) and torch.isinf(s[5, 130]) and torch.isnan(s[7, 0])
        assert torch.isnan(y[[3, 7]]).all() and torch.isnan(y[5, 130])
        assert keep.e[3, 1] == 127 and keep.e[5, 1] == 127 and keep.e[7, 0] == 127 and (keep.e[ok] != 127).all()
        assert (y8.e[3] == 127).all() and y8.e[5, 1] == 127


def test_zero_rows_and_empty(ops):
    z = torch.zeros(3, 300, dtype=BF, device="cuda")
    w = torch.ones(300, device="cuda")
    s, y, rstd, keep, y8 = ops.add_norm(z, z, w, keep=True, out8=True)
    assert (s == 0).all() and (y == 0).all() and (keep.e == -126).all() and (y8.q == 0).all()
    s, y, rstd = ops.add_norm(z[:0], z[:0], w)
    assert s.shape == y.shape == (0, 300) and rstd.shape == (0,)
    dx, dw = ops.add_norm_grad(z[:0], z[:0], s, w, rstd)
    assert dx.shape == (0, 300) and (dw == 0).all()
    base = torch.ones(300, device="cuda")
    ops.add_norm_grad(z[:0], z[:0], s, w, rstd, dweight=base, accumulate=True)
    assert (base == 1).all()


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("t,d", SHAPES)
def test_add_norm_grad(ops, t, d, dt, rt, kept):
    g = gen(t * d + 1)
    ssrc, dsrc, esrc = randn(g, t, d, dtype=rt), randn(g, t, d, dtype=dt), randn(g, t, d, dtype=rt)
    for lead, extra, wt in ((0, 0, dt), (8, 16, F32), (1, 3, BF)):
        w = 1 + randn(g, d, dtype=wt, spread=0.2)
        s, _ = strided(ssrc, lead, extra)
        dy, _ = strided(dsrc, lead, extra)
        ds, _ = strided(esrc, lead, extra)
        rstd = torch.rsqrt(s.float().square().mean(1) + 1e-5)
        act = ops.act_save(s)
        seen = values(act.q, act.e)[:, :d] if kept else s
        given = act if kept else s
        out, buf = strided(torch.zeros(t, d, dtype=rt, device="cuda"), lead, extra)
        dx, dw = ops.add_norm_grad(dy, ds, given, w, rstd, dx=out, dtype=wt)
        assert dx.data_ptr() == out.data_ptr()
        rdx, room, rdw, wroom, _, _ = norm_grad_ref(dy, seen, w, None, rstd)
        rdx = rdx + ds.double()
        within(dx, rdx, room + 4 * U * (rdx.abs() + ds.double().abs()), "dx")
        within(dw, rdw, wroom, "dweight")
        again = ops.add_norm_grad(dy, ds, given, w, rstd, dtype=wt)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
        base = randn(g, d, dtype=wt)
        aw = base.clone()
        # in place
        ds2, _ = strided(esrc, lead, extra)
        dx2, _ = ops.add_norm_grad(dy, ds2, given, w, rstd, dx=ds2, dweight=aw, accumulate=True)
        assert dx2.data_ptr() == ds2.data_ptr() and torch.equal(ds2, dx)
        within(aw, rdw + base.double(), wroom + 2 * U * base.double().abs(), "dweight added")
        dx.fill_(77.0)
        assert (buf == 77.0).all()


def test_grad_of_broadcast_rows(ops):
    """One row of gradients for all tokens (stride 0)."""
    g = gen(4)
    for t, d in ((50, 200), (2000, 1024)):
        s, w = randn(g, t, d), 1 + randn(g, d, spread=0.2)
        dy, ds = randn(g, 1, d).expand(t, d), randn(g, 1, d).expand(t, d)
        rstd = torch.rsqrt(s.square().mean(1) + 1e-5)
        dx, dw = ops.add_norm_grad(dy, ds, s, w, rstd)
        rdx, room, rdw, wroom, _, _ = norm_grad_ref(dy, s, w, None, rstd)
        rdx = rdx + ds.double()
        within(dx, rdx, room + 4 * U * (rdx.abs() + ds.double().abs()), "dx")
        within(dw, rdw, wroom, "dweight")


def test_grad_is_the_derivative(ops):
    """Central differences of sum(dy * y) + sum(dsum * sum) in 64 bits, in x, the residual and the weight."""
    g = gen(22)
    t, d, eps, h = 3, 11, 1e-5, 1e-5
    x, r, w, dy, ds = randn(g, t, d), randn(g, t, d), 1 + randn(g, d, spread=0.2), randn(g, t, d), randn(g, t, d)
    s, _, rstd = ops.add_norm(x, r, w, eps=eps)
    dx, dw = ops.add_norm_grad(dy, ds, s, w, rstd)

    def f(x, r, w):
        s = x + r
        return ((dy.double() * s / (s.square().mean(1, keepdim=True) + eps).sqrt() * w).sum() + (ds.double() * s).sum())
    at = [v.double() for v in (x, r, w)]
    for k, got in ((0, dx), (1, dx), (2, dw)):
        for i in range(got.numel()):
            up, down = [v.clone() for v in at], [v.clone() for v in at]
            up[k].view(-1)[i] += h
            down[k].view(-1)[i] -= h
            # the difference quotient is off by h^2 and by roundings over h, the gradient by some 50 roundings of its terms
            assert abs(float((f(*up) - f(*down)) / (2 * h)) - float(got.view(-1)[i])) < 1e-4


def test_captured_beside_eager(ops):
    g = gen(8)
    for t, d in ((64, 256), (1500, 2048)):
        x, r, w, dy = (randn(g, t, d, dtype=BF) for _ in range(2)), None, 1 + randn(g, d, dtype=BF, spread=0.1), randn(g, t, d, dtype=BF)
        x, r = x
        want = ops.add_norm(x, r, w, keep=True)
        wgrad = ops.add_norm_grad(dy, r, want[3], w, want[2])
        out, total, act = torch.zeros_like(x), torch.zeros_like(x), ops.Act.empty(t, d, "cuda")
        dx, dw = torch.zeros_like(x), torch.zeros(d, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _, _, rstd = ops.add_norm(x, r, w, out=out, sum=total, keep=act)
            ops.add_norm_grad(dy, r, act, w, rstd, dx=dx, dweight=dw)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        for _ in range(3):
            graph.replay()
            with torch.cuda.stream(side):
                eager = ops.add_norm_grad(dy, r, want[3], w, want[2])
        torch.cuda.synchronize()
        assert torch.equal(out, want[1]) and torch.equal(total, want[0]) and torch.equal(dx, wgrad[0]) and torch.equal(dw, wgrad[1])
        assert torch.equal(eager[0], wgrad[0]) and torch.equal(eager[1], wgrad[1])


def test_together_with_the_weight_gradient_and_its_update(ops):
    """A block's step as it is used: the norm's output in 8 bits is the linear layer's kept input, its weight gradient
    goes through the momentum and is made orthogonal, and the stream's gradient comes back through the norm."""
    g = gen(40)
    t, d, n = 1024, 256, 512
    x, r, w = randn(g, t, d, dtype=BF), randn(g, t, d, dtype=BF), 1 + randn(g, d, dtype=BF, spread=0.1)
    weight = randn(g, n, d, dtype=BF, spread=0.06)
    dz, ds = randn(g, t, n, dtype=BF, spread=1e-3), randn(g, t, d, dtype=BF, spread=1e-3)
    s, y, rstd, kept, y8 = ops.add_norm(x, r, w, keep=True, out8=True)
    check_forward(x, r, w, s, y, rstd, kept, y8)
    dweight = ops.weight_grad(dz, y8)
    ref = dz.double().t() @ values(y8.q, y8.e)[:, :d].double()
    assert float((dweight.double() - ref).norm() / ref.norm()) < 1e-6
    m = torch.zeros(n, d, device="cuda")
    update = ops.orthogonalize(dweight, momentum=m)
    u = (dweight.double() * (1 - 0.95) + 0.95 * m.double()).t()
    v = u / u.norm()
    for _ in range(5):
        a = v @ v.t()
        v = 3.4445 * v + (-4.7750 * a + 2.0315 * a @ a) @ v
    assert float((update.double().t() - v).norm() / v.norm()) < 15 * 2.0 ** -12 + 2.0 ** -8
    dy = dz @ weight
    dx, dw = ops.add_norm_grad(dy, ds, kept, w, rstd)
    rdx, room, rdw, wroom, _, _ = norm_grad_ref(dy, values(kept.q, kept.e)[:, :d], w, None, rstd)
    rdx = rdx + ds.double()
    within(dx, rdx, room + 4 * U * (rdx.abs() + ds.double().abs()), "dx")
    within(dw, rdw, wroom, "dweight")


def test_refusals(ops):
    from paper_2609_27193_gb300._abi import LCError
    x, r, w = torch.zeros(4, 64, dtype=BF, device="cuda"), torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    rstd = torch.ones(4, device="cuda")
    for args, kw, error in (((r, x, w), {}, LCError), ((x, r, w), dict(sum=x.clone()), LCError), ((x, r, w), dict(out=r.clone()), LCError),
                            ((x, r[:3], w), {}, ValueError), ((x, r, w[:5]), {}, ValueError), ((x, r, w), dict(out=False), LCError),
                            ((x, r, w), dict(out=x), LCError), ((x, x, w), dict(sum=x), LCError), ((x, r, w), dict(eps=-1.0), LCError),
                            ((x, r.cpu(), w), {}, ValueError), ((x, None, w), {}, TypeError), ((x, r.half(), w), {}, TypeError),
                            ((x, r, w.clone().requires_grad_()), {}, RuntimeError), ((x, r, w), dict(keep=ops.Act.empty(3, 64, "cuda")), ValueError),
                            ((x, r[:, ::2], w), {}, ValueError)):
        with pytest.raises(error):
            ops.add_norm(*args, **kw)
    big = torch.zeros(5, 64, device="cuda")
    with pytest.raises(LCError):
        ops.add_norm(x, big[:4], w, sum=big[1:])
    for args, kw, error in (((x, x, r, w, rstd), {}, LCError), ((r, x, x, w, rstd), {}, LCError), ((x, r, r, w, rstd[:3]), {}, ValueError),
                            ((x, r, r, w, rstd), dict(dx=x.clone()), LCError), ((x, r, r, w, rstd), dict(dx=r[:3]), ValueError),
                            ((x, r.clone(), r, w, rstd), dict(dx=r), LCError), ((x, r, r, w, rstd), dict(accumulate=True), ValueError),
                            ((x, r, ops.Act.empty(4, 65, "cuda"), w, rstd), {}, ValueError), ((x, r, None, w, rstd), {}, TypeError),
                            ((x, r[:3], r, w, rstd), {}, ValueError)):
        with pytest.raises(error):
            ops.add_norm_grad(*args, **kw)


def test_the_c_abi_asks_about_memory(ops):
    """The binding vouches for torch's tensors during its own calls only, whether they succeed or not."""
    from paper_2609_27193_gb300 import _abi
    lib = _abi.load()
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    host = torch.zeros(4, 64).pin_memory()
    rstd, out = torch.zeros(4, device="cuda"), torch.zeros(4, 64, device="cuda")

    def rows(t):
        return _abi.lc_rows(t.data_ptr(), 64, _abi.LC_F32, 0)

    def refused():
        st = lib.lc_add_norm(0, None, rows(x), rows(host), 4, 64, w.data_ptr(), _abi.LC_F32, 1e-5, rows(out), rows(torch.zeros_like(x)),
                             rstd.data_ptr(), None, None)
        assert st == _abi.LC_ERR_INVALID_ARG and b"device memory" in lib.lc_last_error()
    refused()
    ops.add_norm(x, x, w)
    refused()
    with pytest.raises(_abi.LCError):
        ops.add_norm(x, x, w, eps=-1.0)
    refused()
    with pytest.raises(ValueError):
        ops.add_norm(x, host, w)
