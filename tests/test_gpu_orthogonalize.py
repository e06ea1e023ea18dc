"""Updates made orthogonal by Newton-Schulz products, against the definition in 64 bits, in two ways.

Two steps, element by element, against the definition with the operands' roundings (fp16 X, A and B without their
diagonals) made in 64 bits too.  What differs then are fp32 sums: by some 1e-7, which flips the rounding of about one
operand in a thousand by 2^-11 of it.  A flipped element of B (or of A, which comes into B) moves the results of its row by
2^-11 |B| |X|, at most; an element has room for four of the largest such terms and for the sums themselves (SUMS of the
results' root-mean-square), beside half a unit of the output's bf16.  (Each further step turns flips into others: after three the two
sides' roundings are independent, and nothing is learnt from a comparison that the second way does not show.)

All steps, in norm, against the definition itself: three roundings to fp16 a step (X, A, B), each off by at most 2^-12,
and one to bf16, by at most 2^-8.  A step multiplies a disturbance by no more than what it multiplies a small singular
value by, so it grows no faster than the result; added up linearly they are 3 * 2^-12 a step, and 2^-8.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import BF, F32, gen, randn  # noqa: E402

COEF = (3.4445, -4.7750, 2.0315)
SUMS = 1e-5
NEAR = 5 * 3 * 2.0 ** -12 + 2.0 ** -8


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import ops
    return ops


def definition(u, steps=5, coef=COEF, eps=1e-7):
    """In 64 bits; u: [rows, cols]."""
    x = u.double()
    if x.shape[0] > x.shape[1]:
        return definition(u.t(), steps, coef, eps).t()
    every = coef if isinstance(coef[0], tuple) else (coef,) * steps
    x = x / (x.norm() + eps)
    for a, b, c in every:
        g = x @ x.t()
        x = a * x + (b * g + c * g @ g) @ x
    return x


def f16(x, scale):
    return (x * scale).half().double() / scale


def with_roundings(u, steps=5, coef=COEF, eps=1e-7):
    """The same with the operands' roundings.  The scales are powers of two that keep singular values (at most 1.21 with
    these coefficients, 1 to begin with) within half of fp16's range: 2^14 for X and A, and 2^13 for B, whose values reach
    2.81."""
    x = u.double()
    if x.shape[0] > x.shape[1]:
        x, flip = with_roundings(u.t(), steps, coef, eps)
        return x.t(), flip
    sx = min(2.0 ** 14, 2.0 ** math.floor(math.log2(math.sqrt(x.numel()))))
    x = x / (x.norm() + eps)
    a, b, c = coef
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    flip = 0.0
    for _ in range(steps):
        h = f16(x, sx)
        g = h @ h.t()
        d = g.diagonal()
        g0 = f16(g * (1 - eye), 2.0 ** 14)
        sq = g0 @ g0 + (d[:, None] + d[None, :]) * g0 + torch.diag(d * d)
        p = b * (g0 + torch.diag(d)) + c * sq
        p0 = f16(p * (1 - eye), 2.0 ** 13)
        x = (a + p.diagonal())[:, None] * x + p0 @ h
        # (what a step brings along is multiplied by a in the next)
        flip = a * flip + 2.0 ** -11 * float(p0.abs().max() * h.abs().max())
    return x, 4 * flip


def check(call, u, **kw):
    """call(steps): the operator's result for u."""
    got, (ref, flip) = call(2), with_roundings(u, 2, **kw)
    rms = ref.norm() / math.sqrt(ref.numel())
    off = (got.double() - ref).abs()
    bad = off > ref.abs() * 2.0 ** -8 + SUMS * rms + flip
    assert not bad.any(), "%d of %d off, worst %.3g with rms %.3g" % (int(bad.sum()), ref.numel(), float(off.max()), float(rms))
    got, ref = call(5), definition(u, 5, **kw)
    assert float((got.double() - ref).norm() / ref.norm()) < NEAR
    return got


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("m,n", [(1, 2), (2, 1), (3, 64), (64, 64), (65, 63), (100, 257), (128, 128), (129, 128), (128, 1000), (255, 300),
                                 (256, 256), (1024, 256), (515, 1023), (700, 2500), (1023, 1025), (1024, 4096), (3000, 1100), (2100, 2049)])
def test_shapes(ops, dtype, m, n):
    u = randn(gen(m * 7 + n), m, n, dtype=dtype, spread=1e-3)
    got = check(lambda k: ops.orthogonalize(u, steps=k), u)
    assert got.dtype == BF and got.shape == u.shape


def test_one_value(ops):
    """A 1 x 1 matrix: the polynomial five times from 1."""
    for v in (3.0, -0.25):
        got = ops.orthogonalize(torch.full((1, 1), v, device="cuda"))
        assert abs(float(got) - float(definition(torch.tensor([[v]])))) < NEAR


@pytest.mark.parametrize("b,m,n", [(1, 40, 30), (2, 128, 129), (7, 64, 200), (8, 1024, 256), (40, 17, 33), (3, 1100, 1024)])
def test_batches(ops, b, m, n):
    u = randn(gen(b * m), b, m, n)
    u *= torch.logspace(-3, 3, b, device="cuda")[:, None, None] if b > 1 else 1.0
    got = [ops.orthogonalize(u, steps=k) for k in range(6) if k]
    for k in range(b):
        check(lambda steps: got[steps - 1][k], u[k])


@pytest.mark.parametrize("kind", ["decaying", "low", "rows", "one_hot"])
@pytest.mark.parametrize("m,n", [(200, 300), (1024, 1100)])
def test_spectra(ops, kind, m, n):
    """Singular values over orders of magnitude: what a single fp16 number as state would lose."""
    g = gen(m)
    if kind == "decaying":
        q = torch.linalg.qr(torch.randn(m, m, generator=g, device="cuda", dtype=torch.float64))[0]
        v = torch.linalg.qr(torch.randn(n, m, generator=g, device="cuda", dtype=torch.float64))[0]
        u = ((q * (torch.arange(1, m + 1, device="cuda").double() ** -1.5)) @ v.t()).float()
    elif kind == "low":
        u = randn(g, m, 8) @ randn(g, 8, n) + 1e-4 * randn(g, m, n)
    elif kind == "rows":
        u = randn(g, m, n) * torch.exp(2 * randn(g, m, 1))
    else:
        u = torch.eye(m, n, device="cuda")
    check(lambda k: ops.orthogonalize(u, steps=k), u)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e25, 1e37])
def test_magnitudes(ops, scale):
    """The norm's squares leave fp32's range on either side."""
    u = randn(gen(3), 70, 90)
    u = u / u.abs().max() * scale
    if scale > 1e-20:
        check(lambda k: ops.orthogonalize(u, steps=k, eps=0.0), u, eps=0.0)
    else:
        # far below eps: X is next to nothing, and so is what comes of it (at most 3.4445^5 times X's norm)
        assert ops.orthogonalize(u).abs().max() <= 485 * 80 * scale / 1e-7
    assert (ops.orthogonalize(u * 0) == 0).all()
    assert torch.isnan(ops.orthogonalize(u * 0, eps=0.0)).all()


@pytest.mark.parametrize("m,n", [(64, 80), (300, 500), (1100, 1200)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
def test_not_finite(ops, what, m, n):
    """One bad value takes its matrix and no other."""
    u = randn(gen(5), 3, m, n)
    want = ops.orthogonalize(u)
    u[1, m // 2, n - 1] = what
    got = ops.orthogonalize(u)
    assert torch.isnan(got[1]).all()
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("m,n", [(60, 100), (100, 60), (1030, 1100)])
def test_strides(ops, dtype, m, n):
    """Rows off 16 bytes, wider rows, every other matrix, matrices between one another's rows; what lies around an
    output stays."""
    u = randn(gen(9), 4, m, n, dtype=dtype)
    want = ops.orthogonalize(u[::2].contiguous())
    assert torch.equal(ops.orthogonalize(u[::2]), want)
    for lead, extra in ((1, 0), (3, 5), (8, 8)):
        buf = torch.zeros(lead + 2 * m * (n + extra), dtype=dtype, device="cuda")
        v = buf[lead:].view(2, m, n + extra)[:, :, :n]
        v.copy_(u[::2])
        obuf = torch.full((lead + 2 * m * (n + extra),), 7.0, dtype=BF, device="cuda")
        o = obuf[lead:].view(2, m, n + extra)[:, :, :n]
        assert ops.orthogonalize(v, out=o).data_ptr() == o.data_ptr()
        for k in range(2):
            check(lambda steps: ops.orthogonalize(v, steps=steps, out=o)[k], u[2 * k])
        o.fill_(7.0)
        assert (obuf == 7.0).all()
    between = torch.empty(m, 2, n, dtype=BF, device="cuda")
    got = ops.orthogonalize(u[::2], out=between.transpose(0, 1))
    assert torch.equal(between[:, 0], want[0]) and torch.equal(between[:, 1], want[1])
    one = u[:1, :1]
    assert ops.orthogonalize(one[:, :, :1]).shape == (1, 1, 1)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(50, 70), (3, 70, 50), (515, 1023), (1200, 1100)])
def test_momentum(ops, dtype, nesterov, shape):
    """momentum: two fp32 operations on it, each off by 2^-24 of what goes in."""
    g = gen(sum(shape))
    u, m0 = randn(g, *shape, dtype=dtype), randn(g, *shape)
    m = m0.clone()
    beta = 0.9
    version = m._version
    got = ops.orthogonalize(u, momentum=m, beta=beta, nesterov=nesterov)
    assert m._version > version
    ref = m0.double() + (1 - beta) * (u.double() - m0.double())
    assert ((m.double() - ref).abs() <= 4 * 2.0 ** -24 * (m0.double().abs() + u.double().abs())).all()
    up = u.double() + beta * (ref - u.double()) if nesterov else ref
    up = up.reshape(-1, *shape[-2:])
    two = ops.orthogonalize(u, momentum=m0.clone(), beta=beta, nesterov=nesterov, steps=2)
    for k in range(len(up)):
        check(lambda steps: (two if steps == 2 else got).reshape(-1, *shape[-2:])[k], up[k])
    # strided momentum, an update whose rows are off 16 bytes
    if len(shape) == 2:
        buf = torch.zeros(shape[0], shape[1] + 3, device="cuda")
        v = buf[:, 1:1 + shape[1]]
        v.copy_(m0)
        ops.orthogonalize(u, momentum=v, beta=beta, nesterov=nesterov)
        assert torch.equal(v, m) and (buf[:, 0] == 0).all() and (buf[:, -2:] == 0).all()


def test_coefficients(ops):
    """Other polynomials, one a step, more and fewer steps."""
    u = randn(gen(1), 90, 130)
    cubic = (1.5, -0.5, 0.0)
    for steps, coef in ((1, COEF), (3, cubic), (12, cubic), (16, (1.875, -1.25, 0.375)), (2, ((3.4445, -4.775, 2.0315), cubic))):
        got = ops.orthogonalize(u, steps=steps, coefficients=coef)
        ref = definition(u, steps, coef)
        assert float((got.double() - ref).norm() / ref.norm()) < 3 * steps * 2.0 ** -12 + 2.0 ** -8, (steps, coef)
    assert torch.equal(ops.orthogonalize(u, steps=2, coefficients=[[3.4445, -4.775, 2.0315], [1.5, -0.5, 0.0]]),
                       ops.orthogonalize(u, steps=2, coefficients=((3.4445, -4.775, 2.0315), cubic)))
    # cubic steps until they stand still: U V^T of the singular value decomposition
    got = ops.orthogonalize(randn(gen(2), 64, 512), steps=16, coefficients=cubic).double()
    assert (got @ got.t() - torch.eye(64, device="cuda")).abs().max() < 0.02


@pytest.mark.parametrize("shape", [(200, 190), (8, 256, 512), (1024, 1024)])
def test_same_bits(ops, shape):
    """The same call gives the same bits, whatever the scratch held, captured or not."""
    u, m = randn(gen(4), *shape), randn(gen(5), *shape)
    first = ops.orthogonalize(u, momentum=m.clone())
    other = ops.orthogonalize(randn(gen(6), *shape))
    for _ in range(3):
        assert torch.equal(ops.orthogonalize(u, momentum=m.clone()), first)
    out, mm = torch.empty_like(first), m.clone()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.orthogonalize(u, momentum=mm, out=out)
    u2, out2 = randn(gen(6), *shape), torch.empty_like(first)
    with torch.cuda.graph(second):
        ops.orthogonalize(u2, out=out2)
    for _ in range(2):
        mm.copy_(m)
        out.zero_()
        graph.replay()
        second.replay()
        assert torch.equal(out, first) and torch.equal(out2, other)


def test_streams_beside_one_another(ops):
    """Calls on three streams at once: each launch is as large as the device."""
    us = [randn(gen(k), 1024, 1100 + 100 * k) for k in range(3)] + [randn(gen(9), 200, 200)]
    want = [ops.orthogonalize(u) for u in us]
    streams = [torch.cuda.Stream() for _ in us]
    torch.cuda.synchronize()
    got = [[] for _ in us]
    for _ in range(5):
        for k, (s, u) in enumerate(zip(streams, us)):
            with torch.cuda.stream(s):
                got[k].append(ops.orthogonalize(u))
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for xs, w in zip(got, want) for x in xs)


def test_refusals(ops):
    from paper_2609_27193_gb300._abi import LCError
    u = randn(gen(1), 64, 96)
    o = torch.empty(64, 96, dtype=BF, device="cuda")
    for kw, error in ((dict(momentum=torch.zeros(64, 95, device="cuda")), ValueError), (dict(momentum=o), TypeError),
                      (dict(out=u), TypeError), (dict(out=o[:63]), ValueError), (dict(steps=0), ValueError),
                      (dict(steps=17), ValueError), (dict(coefficients=(1.0, 2.0)), ValueError),
                      (dict(steps=3, coefficients=((1.0, 0.0, 0.0),) * 2), ValueError), (dict(eps=-1.0), LCError),
                      (dict(coefficients=(1e4, 0.0, 0.0)), LCError), (dict(coefficients=(9.0, 0.0, 0.0)), LCError),
                      (dict(coefficients=(float("nan"), 0.0, 0.0)), LCError), (dict(momentum=u), LCError),
                      (dict(momentum=torch.zeros(64, 96, device="cuda"), beta=1.0), LCError),
                      (dict(out=torch.empty(96, dtype=BF, device="cuda").expand(64, 96)), LCError),
                      (dict(out=torch.empty(96, 64, dtype=BF, device="cuda").t()), ValueError)):
        with pytest.raises(error):
            ops.orthogonalize(u, **kw)
    for bad, error in ((u.half(), TypeError), (u.cpu(), ValueError), (u[0], ValueError), (u.t(), ValueError),
                       (u[:, :0], ValueError), (u[None, None], ValueError), (u.clone().requires_grad_(), RuntimeError)):
        with pytest.raises(error):
            ops.orthogonalize(bad)
    assert ops.orthogonalize(u[None][:0]).shape == (0, 64, 96)
    with torch.no_grad():
        ops.orthogonalize(u.clone().requires_grad_())
    both = torch.zeros(128, 96, dtype=BF, device="cuda")
    with pytest.raises(LCError):
        ops.orthogonalize(both[:64], out=both[32:96])
