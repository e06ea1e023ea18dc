"""The operators of a training step (embedding, norm, 8-bit activations, the
weight gradient) against their definitions in 64 bits.

Bounds come from the arithmetic, element by element: a sum of n fp32 terms is
off by at most n * 2^-24 of the sum of their magnitudes, each further fp32
operation adds 2^-24 of its result, and a bf16 output half a unit of 8 bits.
What is exact (copies, the checkpoint) is compared for equality.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import ops
    return ops


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32, spread=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * spread).to(dtype)


def strided(x, lead, extra):
    """x's values in rows that start `lead` elements into a buffer and lie `extra` further apart than needed."""
    t, d = x.shape
    buf = torch.full((lead + t * (d + extra) + 8,), 77.0, dtype=x.dtype, device=x.device)
    v = buf[lead:lead + t * (d + extra)].view(t, d + extra)[:, :d]
    v.copy_(x)
    return v, buf


def within(got, ref, bound, what):
    """|got - ref| <= bound (+ the rounding of got's type), NaN where ref is."""
    got64 = got.double()
    assert torch.equal(torch.isnan(got64), torch.isnan(ref)), what + ": NaN in other places"
    room = bound + (ref.abs() * 2.0 ** -8 if got.dtype == BF else ref.abs() * U) + 1e-37
    off = (got64 - ref).abs()
    bad = (off > room) & ~torch.isnan(ref)
    assert not bad.any(), "%s: %d of %d off, worst %.3g with %.3g allowed" % (
        what, int(bad.sum()), ref.numel(), float((off - room)[bad].max()), float(room[bad].max()))


# --- embedding -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t,v,d", [(1, 1, 1), (1, 50, 256), (7, 33, 129), (64, 1000, 768), (513, 4099, 1026), (300, 9, 8200)])
def test_embed(ops, dtype, t, v, d):
    g = gen(t + d)
    table = randn(g, v, d, dtype=dtype)
    ids = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32 if d % 2 else torch.int64)
    if t > 4:
        ids[2], ids[3], ids[4] = -1, v, -(2 ** 31)
    y = ops.embed(table, ids, scale=27.5)
    ok = (ids >= 0) & (ids < v)
    ref = (table[ids.clamp(0, v - 1).long()].float() * 27.5).to(dtype)
    ref[ids < 0] = 0
    assert torch.equal(y[ids < v], ref[ids < v])
    assert torch.isnan(y[ids >= v]).all()
    assert torch.equal(ops.embed(table, ids)[ok], table[ids[ok].long()])


@pytest.mark.parametrize("lead,extra", [(0, 8), (1, 3), (8, 0), (3, 5)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_embed_strides(ops, dtype, lead, extra):
    g = gen(5)
    t, v, d = 37, 61, 200
    table, _ = strided(randn(g, v, d, dtype=dtype), lead, extra)
    ids = torch.randint(0, v, (t,), generator=g, device="cuda")
    out, buf = strided(torch.zeros(t, d, dtype=dtype, device="cuda"), extra, lead)
    ops.embed(table, ids, out=out)
    assert torch.equal(out, table[ids])
    out.fill_(77.0)
    assert (buf == 77.0).all()     # nothing between the rows was touched


def test_embed_past_32_bits(ops):
    """Rows whose element offset does not fit 32 bits."""
    v, d = 1_100_000, 2048
    table = torch.zeros(v, d, dtype=BF, device="cuda")
    ids = torch.tensor([v - 1, 0, 1_050_001, 1_048_576, 524_288], device="cuda")
    table[ids] = torch.arange(1, 6, device="cuda", dtype=BF)[:, None]
    assert torch.equal(ops.embed(table, ids), table[ids])
    dy = torch.ones(5, d, dtype=BF, device="cuda")
    grad = ops.embed_grad(dy, ids, v)
    assert torch.equal(grad[ids], dy) and int((grad[:, 0] != 0).sum()) == 5 and int((grad[:, -1] != 0).sum()) == 5


def embed_grad_ref(dy, ids, v, scale, skip=-1, base=None):
    d = dy.shape[1]
    ref = torch.zeros(v + 1, d, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(ref)
    n = torch.zeros(v + 1, device="cuda", dtype=torch.float64)
    row = torch.where((ids < 0) | (ids >= v) | (ids == skip), v, ids).long()
    ref.index_add_(0, row, dy.double())
    mag.index_add_(0, row, dy.double().abs())
    n.index_add_(0, row, torch.ones_like(row, dtype=torch.float64))
    ref, mag, n = ref[:v] * scale, mag[:v] * abs(scale), n[:v]
    if base is not None:
        ref, mag = ref + base.double(), mag + base.double().abs()
    return ref, (n[:, None] + 3) * U * mag, n


IDS = ["spread", "same", "few", "masked", "word"]


def make_ids(g, t, v, how):
    if how == "spread":
        return torch.randint(0, v, (t,), generator=g, device="cuda")
    if how == "same":
        return torch.full((t,), v - 1, device="cuda")
    if how == "few":
        return torch.randint(0, min(v, 3), (t,), generator=g, device="cuda") * max(1, v // 3)
    if how == "masked":
        return torch.full((t,), -1, device="cuda")
    u = torch.rand(t, generator=g, device="cuda")
    ids = (float(v) ** u - 1).long().clamp(0, v - 1)
    ids[torch.rand(t, generator=g, device="cuda") < 0.1] = -1
    return ids


@pytest.mark.parametrize("how", IDS)
@pytest.mark.parametrize("t,v,d,dt,gt", [
    (1, 1, 1, F32, F32), (1, 511, 64, BF, F32), (33, 512, 129, BF, BF), (64, 70, 2048, BF, F32), (63, 9, 1001, F32, F32),
    (17, 3000, 520, F32, BF), (65, 70, 200, BF, BF), (777, 513, 256, F32, BF),
    (2048, 8000, 256, BF, F32), (2049, 131072, 24, F32, F32), (20011, 40, 1030, BF, BF), (5000, 262145, 8, BF, F32), (8193, 600, 64, F32, F32), (65536, 128256, 8, BF, BF),
    (70001, 300, 8, BF, F32), (140000, 70000, 16, BF, F32)])
def test_embed_grad(ops, how, t, v, d, dt, gt):
    g = gen(t + v)
    dy = randn(g, t, d, dtype=dt)
    ids = make_ids(g, t, v, how)
    if d % 2 == 0:
        ids = ids.int()
    grad = torch.full((v, d), math.nan, dtype=gt, device="cuda")
    ops.embed_grad(dy, ids, scale=0.75, grad=grad)
    ref, bound, n = embed_grad_ref(dy, ids, v, 0.75)
    within(grad, ref, bound, "grad")
    assert (grad[n == 0] == 0).all()
    again = ops.embed_grad(dy, ids, v, scale=0.75, dtype=gt)
    assert torch.equal(again, grad)                      # the same bits every time


@pytest.mark.parametrize("gt", [BF, F32])
@pytest.mark.parametrize("t", [50, 700])
def test_embed_grad_accumulate_skip_and_errors_in_ids(ops, t, gt):
    g = gen(11)
    v, d = 90, 136
    dy = randn(g, t, d, dtype=BF)
    ids = torch.randint(0, v, (t,), generator=g, device="cuda")
    ids[5], ids[6], ids[7] = -7, v, v + 1000
    base = randn(g, v, d, dtype=gt)
    grad = base.clone()
    ops.embed_grad(dy, ids, scale=2.0, grad=grad, skip_id=3, accumulate=True)
    ref, bound, n = embed_grad_ref(dy, ids, v, 2.0, skip=3, base=base)
    within(grad, ref, bound, "grad")
    assert torch.equal(grad[n == 0], base[n == 0]) and n[3] == 0


@pytest.mark.parametrize("dt,gt", [(BF, F32), (F32, BF), (BF, BF)])
@pytest.mark.parametrize("t", [40, 500])
def test_embed_grad_strides(ops, t, dt, gt):
    g = gen(12)
    v, d = 70, 200
    ids = torch.randint(0, v, (t,), generator=g, device="cuda")
    src = randn(g, t, d, dtype=dt)
    want = ops.embed_grad(src, ids, v, dtype=gt)
    for lead, extra in ((0, 8), (1, 0), (8, 16), (3, 5)):
        dy, _ = strided(src, lead, extra)
        grad, buf = strided(torch.zeros(v, d, dtype=gt, device="cuda"), lead, extra)
        ops.embed_grad(dy, ids, grad=grad)
        ref, bound, _ = embed_grad_ref(src, ids, v, 1.0)
        within(grad, ref, bound, "grad")
        grad.fill_(77.0)
        assert (buf == 77.0).all()
    one = src[:1].expand(t, d)                           # a broadcast gradient: stride 0
    within(ops.embed_grad(one, ids, v, dtype=gt), *embed_grad_ref(one, ids, v, 1.0)[:2], "expanded")
    assert want.shape == (v, d)


def test_embed_grad_nothing(ops):
    dy = torch.empty(0, 16, dtype=BF, device="cuda")
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    assert (ops.embed_grad(dy, ids, 10) == 0).all()
    base = torch.ones(10, 16, device="cuda")
    assert (ops.embed_grad(dy, ids, grad=base, accumulate=True) == 1).all()
    assert ops.embed(base, ids).shape == (0, 16)


def test_embed_grad_of_a_nan_stays_in_its_row(ops):
    dy = torch.ones(64, 32, device="cuda")
    dy[7, 3] = math.nan
    dy[9, 4] = math.inf
    ids = torch.arange(64, device="cuda") % 16
    grad = ops.embed_grad(dy, ids, 20)
    assert torch.isnan(grad[7, 3]) and torch.isinf(grad[9, 4])
    assert int((~torch.isfinite(grad)).sum()) == 2


def test_embed_grad_is_the_derivative(ops):
    """Central differences of sum(dy * embed) in 64 bits."""
    g = gen(13)
    t, v, d = 40, 12, 5
    table = randn(g, v, d).double()
    ids = torch.randint(0, v, (t,), generator=g, device="cuda")
    dy = randn(g, t, d)
    grad = ops.embed_grad(dy, ids, v, scale=3.0)

    def loss(e):
        return float((dy.double() * (3.0 * e[ids])).sum())
    h = 1e-3
    for r in range(v):
        for c in range(d):
            up, down = table.clone(), table.clone()
            up[r, c] += h
            down[r, c] -= h
            # linear, so only the differences' own rounding: 64 bits of a sum of 200 terms over h
            assert abs((loss(up) - loss(down)) / (2 * h) - float(grad[r, c])) < 1e-4


# --- 8-bit activations -----------------------------------------------------------------------------------------

POW2 = torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64)


def pow2(e):
    return POW2.cuda()[e.long() + 200]


def quantize(x):
    """The definition, in 64 bits and whole blocks."""
    t, d = x.shape
    nb = -(-d // 128)
    v = torch.zeros(t, nb * 128, dtype=torch.float64, device="cuda")
    v[:, :d] = x.double()
    v = v.view(t, nb, 128)
    bad = ~torch.isfinite(v).all(2)
    a = torch.where(torch.isfinite(v), v, 0).abs().amax(2)
    m, k = torch.frexp(a)
    e = torch.where(m <= 127 / 128, k - 7, k - 6).clamp(min=-126)
    e = torch.where(a == 0, -126, e).clamp(max=121)
    q = torch.round(v * pow2(-e)[:, :, None]).clamp(-127, 127)
    q[bad] = 0
    return q.to(torch.int8).view(t, nb * 128), torch.where(bad, 127, e).to(torch.int8), bad


def values(q, e):
    t, nb = e.shape
    v = q.view(t, nb, 128).double() * pow2(e)[:, :, None]
    v[e == 127] = math.nan
    return v.reshape(t, nb * 128)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t,d", [(1, 1), (3, 127), (5, 128), (2, 129), (17, 1000), (64, 4096), (3, 14337), (2051, 256)])
@pytest.mark.parametrize("lead,extra", [(0, 0), (1, 2)])
def test_act(ops, dtype, t, d, lead, extra):
    g = gen(t + d)
    x = randn(g, t, d, dtype=dtype) * torch.exp2(torch.randint(-20, 20, (t, 1), generator=g, device="cuda").to(dtype))
    x[0, 0] = 127.0                                       # a block that ends on a step, one a step above
    if d > 128:
        x[0, 128] = 127.5
    x, _ = strided(x.to(dtype), lead, extra)
    a = ops.act_save(x)
    q, e, _ = quantize(x)
    assert torch.equal(a.e, e) and torch.equal(a.q, q)
    for out in (BF, F32):
        y, buf = strided(torch.zeros(t, d, dtype=out, device="cuda"), lead, extra)
        ops.act_load(a, out=y)
        assert torch.equal(y.double(), values(q, e)[:, :d])
        y.fill_(77.0)
        assert (buf == 77.0).all()
    # half a step of the block is the most a value moves
    step = pow2(e).repeat_interleave(128, 1)[:, :d]
    assert ((values(q, e)[:, :d] - x.double()).abs() <= step / 2).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_act_extremes(ops, dtype):
    big = torch.finfo(dtype).max
    x = torch.zeros(8, 384, dtype=dtype, device="cuda")
    x[0, 5] = big
    x[1, 5], x[1, 130] = math.nan, 1.0
    x[2, 200], x[2, 1] = -math.inf, 3.0
    x[3, 7] = 2.0 ** -126
    x[4, 9] = torch.finfo(dtype).tiny / 64                # subnormal
    x[5, :] = -big
    x[6, 383] = -(2.0 ** -133)
    q, e, bad = quantize(x)
    for lead in (0, 1):
        v, _ = strided(x, lead, lead)
        a = ops.act_save(v)
        assert torch.equal(a.q, q) and torch.equal(a.e, e)
        y = ops.act_load(a, dtype=dtype)
        assert torch.equal(torch.isnan(y).view(8, 3, 128).all(2), bad) and int(torch.isnan(y).sum()) == 128 * int(bad.sum())
        assert int(bad.sum()) == 2
        fine = ~torch.isnan(y)
        assert torch.equal(y[fine].double(), values(q, e)[fine])


# --- norm ------------------------------------------------------------------------------------------------------

NORMS = [(1, 1, F32, F32), (3, 5, BF, F32), (9, 127, BF, BF), (130, 256, F32, F32), (65, 768, BF, BF),
         (33, 1000, BF, F32), (40, 2048, BF, BF), (17, 2049, F32, BF), (12, 4096, BF, BF), (7, 5000, F32, F32),
         (5, 8192, BF, F32), (6, 9001, BF, BF), (3, 16384, F32, F32), (4, 16384, BF, BF), (1500, 64, BF, BF)]
SUMS = 96       # the most terms that one fp32 chain of a row's sums has: in a thread, in a warp, over the warps


def norm_ref(x, w, b, kind, eps):
    x = x.double()
    mean = x.mean(1) if kind == "layer" else None
    c = x if mean is None else x - mean[:, None]
    rstd = 1 / ((c * c).mean(1) + eps).sqrt()
    y = c * rstd[:, None] * w.double()
    return y if b is None else y + b.double(), mean, rstd, c * rstd[:, None]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("t,d,dt,wt", NORMS)
def test_norm(ops, kind, t, d, dt, wt):
    g = gen(t * d)
    shift = 3.0 if kind == "layer" else 0.0
    src = randn(g, t, d) + shift
    w = 1 + randn(g, d, dtype=wt, spread=0.2)
    b = randn(g, d, dtype=wt) if kind == "layer" else None
    for lead, extra in ((0, 0), (0, 8), (1, 2)):
        x, _ = strided(src.to(dt), lead, extra)
        out, buf = strided(torch.zeros(t, d, dtype=dt, device="cuda"), lead, extra)
        y, mean, rstd, keep = ops.norm(x, w, b, eps=1e-5, kind=kind, out=out, keep=True)
        ref, rmean, rrstd, xhat = norm_ref(x, w, b, kind, 1e-5)
        a = x.double().abs().mean(1)
        if mean is not None:
            within(mean, rmean, SUMS * U * a, "mean")
        else:
            assert rmean is None
        # the variance moves by twice its own chain, and rstd by half of that; 4 for rsqrt and the epsilon
        within(rstd, rrstd, (SUMS + 4) * U * rrstd, "rstd")
        room = ((SUMS + 8) * U * xhat.abs() + (SUMS + 8) * U * (a * rrstd)[:, None]) * w.double().abs()
        within(y, ref, room + (4 * U * b.double().abs() if b is not None else 0), "y")
        q, e, _ = quantize(x)
        assert torch.equal(keep.q, q) and torch.equal(keep.e, e)
        y.fill_(77.0)
        assert (buf == 77.0).all()


def norm_grad_ref(dy, x, w, mean, rstd):
    h = (x.double() if mean is None else x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    dy, w = dy.double(), w.double()
    a = dy * w
    m1 = a.mean(1, keepdim=True) if mean is not None else 0.0
    m2 = (a * h).mean(1, keepdim=True)
    r = rstd.double()[:, None]
    dx = r * (a - m1 - h * m2)
    # h is off by 3 roundings of x - mean and the product
    hb = 3 * U * ((x.double().abs() + (0 if mean is None else mean.double().abs()[:, None])) * r)
    room = r * (4 * U * a.abs() + (SUMS + 4) * U * a.abs().mean(1, keepdim=True)
                + (SUMS + 8) * U * h.abs() * (a * h).abs().mean(1, keepdim=True)
                + hb * m2.abs() + h.abs() * (a.abs() * hb).mean(1, keepdim=True)) + 4 * U * dx.abs()
    t = dy.shape[0]
    return dx, room, (dy * h).sum(0), ((t + 16) * U * (dy * h).abs().sum(0) + (dy.abs() * hb).sum(0)), dy.sum(0), \
        (t + 16) * U * dy.abs().sum(0)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("t,d,dt,wt", NORMS)
def test_norm_grad(ops, kept, kind, t, d, dt, wt):
    g = gen(t * d + 1)
    src = randn(g, t, d) + (1.0 if kind == "layer" else 0.0)
    dsrc = randn(g, t, d)
    w = 1 + randn(g, d, dtype=wt, spread=0.2)
    for lead, extra in ((0, 0), (0, 8), (1, 2)):
        x, _ = strided(src.to(dt), lead, extra)
        dy, _ = strided(dsrc.to(dt), lead, extra)
        _, mean, rstd, keep = ops.norm(x, w, None, kind=kind, keep=True)
        seen = values(keep.q, keep.e)[:, :d] if kept else x
        dxb, buf = strided(torch.zeros(t, d, dtype=dt, device="cuda"), lead, extra)
        dx, dw, db = ops.norm_grad(dy, keep if kept else x, w, mean, rstd, bias=True, dx=dxb, dtype=wt)
        rdx, room, rdw, wroom, rdb, broom = norm_grad_ref(dy, seen, w, mean, rstd)
        within(dx, rdx, room, "dx")
        within(dw, rdw, wroom, "dweight")
        within(db, rdb, broom, "dbias")
        again = ops.norm_grad(dy, keep if kept else x, w, mean, rstd, bias=True, dtype=wt)
        assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))
        base_w, base_b = randn(g, d, dtype=wt), randn(g, d, dtype=wt)
        aw, ab = base_w.clone(), base_b.clone()
        ops.norm_grad(dy, keep if kept else x, w, mean, rstd, dweight=aw, dbias=ab, accumulate=True)
        within(aw, rdw + base_w.double(), wroom + 2 * U * base_w.double().abs(), "dweight added")
        within(ab, rdb + base_b.double(), broom + 2 * U * base_b.double().abs(), "dbias added")
        dx.fill_(77.0)
        assert (buf == 77.0).all()


def test_norm_grad_long(ops):
    """More rows than the device holds CTAs, and a broadcast gradient."""
    g = gen(21)
    t, d = 5003, 384
    x = randn(g, t, d, dtype=BF)
    w = 1 + randn(g, d, dtype=BF, spread=0.2)
    dy = randn(g, 1, d, dtype=BF).expand(t, d)
    _, mean, rstd = ops.norm(x, w, None)
    dx, dw, db = ops.norm_grad(dy, x, w, mean, rstd, bias=True)
    rdx, room, rdw, wroom, rdb, broom = norm_grad_ref(dy, x, w, mean, rstd)
    within(dx, rdx, room, "dx")
    within(dw, rdw, wroom, "dweight")
    within(db, rdb, broom, "dbias")


MANY = [(617, 40, BF, BF), (5000, 64, F32, F32), (613, 256, F32, F32), (640, 520, BF, F32), (3001, 768, BF, BF),
        (611, 1024, BF, BF), (1300, 2048, BF, BF), (620, 4096, BF, F32), (609, 4096, F32, BF), (612, 6000, BF, BF),
        (610, 8192, F32, F32), (625, 12296, BF, BF), (610, 16384, BF, BF), (615, 16384, F32, F32)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("t,d,dt,wt", MANY)
def test_norm_of_many_rows(ops, kind, t, d, dt, wt):
    """Enough rows to stream through shared memory; rows of a wider buffer too; a NaN stays in its row."""
    g = gen(t * d)
    shift = 2.0 if kind == "layer" else 0.0
    src = (randn(g, t, d) + shift).to(dt)
    src[t // 2, d // 3] = math.nan
    w = 1 + randn(g, d, dtype=wt, spread=0.2)
    b = randn(g, d, dtype=wt) if kind == "layer" else None
    dsrc = randn(g, t, d, dtype=dt)
    for extra in (0, 16):
        x, _ = strided(src, 0, extra)
        dy, _ = strided(dsrc, 8, extra)
        y, mean, rstd, keep = ops.norm(x, w, b, kind=kind, keep=True)
        ref, rmean, rrstd, xhat = norm_ref(x, w, b, kind, 1e-5)
        a = x.double().abs().mean(1)
        if mean is not None:
            within(mean, rmean, SUMS * U * a, "mean")
        within(rstd, rrstd, (SUMS + 4) * U * rrstd, "rstd")
        room = ((SUMS + 8) * U * xhat.abs() + (SUMS + 8) * U * (a * rrstd)[:, None]) * w.double().abs()
        within(y, ref, room + (4 * U * b.double().abs() if b is not None else 0), "y")
        q, e, _ = quantize(x)
        assert torch.equal(keep.q, q) and torch.equal(keep.e, e)
        assert torch.equal(ops.norm(x, w, b, kind=kind)[0].isnan().any(1), x.isnan().any(1))
        # gradients: from the rows without the NaN, whole
        ok = ~x.isnan().any(1)
        stat = rstd.clone()
        stat[~ok] = 1.0
        mu = None if mean is None else torch.where(ok, mean, 0.0)
        for kept in (False, True):
            seen = values(keep.q, keep.e)[:, :d] if kept else x
            dx, dw, db = ops.norm_grad(dy, keep if kept else x, w, mu, stat, bias=True)
            assert torch.isnan(dx[t // 2]).any() and torch.isfinite(dx[ok]).all()
            rdx, room, rdw, wroom, rdb, broom = norm_grad_ref(dy[ok], seen[ok], w, None if mu is None else mu[ok], stat[ok])
            within(dx[ok], rdx, room, "dx")
            within(db, dsrc.double().sum(0), (t + 16) * U * dsrc.double().abs().sum(0), "dbias")
            bad = torch.isnan(dw)
            assert bad[d // 3] and int(bad.sum()) <= (128 if kept else 1)
            src2 = torch.where(seen.isnan(), 0.0, seen.double())
            h = (src2 if mu is None else torch.where(seen.isnan(), 0.0, src2 - mu.double()[:, None])) * stat.double()[:, None]
            full = (dsrc.double() * h).sum(0)
            within(dw[~bad], full[~bad], ((t + 16) * U * (dsrc.double() * h).abs().sum(0) + 6 * U * (
                dsrc.double().abs() * (src2.abs() + shift + 1) * stat.double()[:, None]).sum(0))[~bad], "dweight")
            again = ops.norm_grad(dy, keep if kept else x, w, mu, stat, bias=True)
            assert torch.equal(again[0][ok], dx[ok]) and torch.equal(again[1][~bad], dw[~bad]) and torch.equal(again[2], db)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_grad_is_the_derivative(ops, kind):
    """Central differences of sum(dy * norm) in 64 bits."""
    g = gen(22)
    t, d, eps, h = 3, 11, 1e-5, 1e-5
    x, w, b, dy = randn(g, t, d), 1 + randn(g, d, spread=0.2), randn(g, d), randn(g, t, d)
    _, mean, rstd = ops.norm(x, w, b, eps=eps, kind=kind)
    dx, dw, db = ops.norm_grad(dy, x, w, mean, rstd, bias=True)

    def slope(which, i):
        out = []
        for s in (h, -h):
            p = [x.double().clone(), w.double().clone(), b.double().clone()]
            p[which].view(-1)[i] += s
            out.append(float((dy.double() * norm_ref(p[0], p[1], p[2], kind, eps)[0]).sum()))
        return (out[0] - out[1]) / (2 * h)
    # the differences are off by h^2 of third derivatives and 2^-52 / h of the sums; fp32 chains of 2^-24 * SUMS
    for which, got in ((0, dx), (1, dw), (2, db)):
        for i in range(got.numel()):
            assert abs(slope(which, i) - float(got.view(-1)[i])) < 2e-4


def test_norm_non_finite_rows_stay_alone(ops):
    g = gen(23)
    x = randn(g, 6, 500, dtype=BF)
    x[1, 3], x[4, 200] = math.nan, math.inf
    w = torch.ones(500, dtype=BF, device="cuda")
    y, mean, rstd = ops.norm(x, w)
    assert torch.isnan(y[1]).all() and torch.isnan(y[4]).any()
    fine = [0, 2, 3, 5]
    assert torch.isfinite(y[fine]).all()
    z, _, _ = ops.norm(torch.zeros(2, 500, device="cuda"), w)
    assert (z == 0).all()                                  # epsilon keeps a constant row finite


def test_norm_nothing(ops):
    x = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    y, mean, rstd = ops.norm(x, w)
    assert y.shape == (0, 64) and mean.numel() == 0
    _, dw, db = ops.norm_grad(y, x, w, mean, rstd, bias=True)
    assert (dw == 0).all() and (db == 0).all()
    base = torch.ones(64, device="cuda")
    ops.norm_grad(y, x, w, mean, rstd, dweight=base, accumulate=True)
    assert (base == 1).all()


# --- weight gradient -------------------------------------------------------------------------------------------

WGRADS = [(1, 1, 1), (1, 300, 200), (2, 64, 130), (15, 128, 128), (16, 129, 257), (63, 256, 128), (64, 100, 640),
          (65, 512, 256), (200, 33, 1000), (1000, 257, 129), (513, 768, 768), (4099, 128, 384), (2048, 1024, 256)]


def wgrad_ref(dy, a):
    x = values(a.q, a.e)[:, :a.dim]
    dy = dy.double()
    parts = 3
    ref = dy.t() @ x
    mag = dy.abs().t() @ x.abs()
    # chains of at most 3 products a token (a 32-bit gradient comes in three parts); the accumulator may cut off
    # instead of rounding: 2^-23
    return ref, (parts * dy.shape[0] + 16) * 2 * U * mag


@pytest.mark.parametrize("dt,gt", [(BF, F32), (BF, BF), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("t,n,k", WGRADS)
def test_weight_grad(ops, dt, gt, t, n, k):
    g = gen(t + n + k)
    a = ops.act_save(randn(g, t, k, dtype=dt))
    src = randn(g, t, n, dtype=dt)
    ref, room = wgrad_ref(src, a)
    for lead, extra in ((0, 0), (0, 8), (1, 3)):
        dy, _ = strided(src, lead, extra)
        out, buf = strided(torch.full((n, k), math.nan, dtype=gt, device="cuda"), lead, extra)
        dw = ops.weight_grad(dy, a, grad=out)
        within(dw, ref, room, "dw")
        first = dw.clone()
        ops.weight_grad(dy, a, grad=out)
        assert torch.equal(first, out)
        base = randn(g, n, k, dtype=gt)
        out.copy_(base)
        ops.weight_grad(dy, a, grad=out, accumulate=True)
        within(out, ref + base.double(), room + 2 * U * base.double().abs(), "dw added")
        out.fill_(77.0)
        assert (buf == 77.0).all()


def test_weight_grad_broadcast_and_checkpoint_views(ops):
    """A gradient with stride 0, and a checkpoint inside a larger buffer."""
    g = gen(31)
    t, n, k = 300, 96, 200
    x = randn(g, t, k, dtype=BF)
    big = ops.Act.empty(t, 900, "cuda")
    view = ops.Act(big.q[:, 128:512], big.e[:, 1:4], k)
    ops.act_save(x, view)
    dy = randn(g, 1, n, dtype=BF).expand(t, n)
    ref, room = wgrad_ref(dy, ops.act_save(x))
    within(ops.weight_grad(dy, view), ref, room, "dw")
    assert torch.equal(ops.act_load(view), ops.act_load(ops.act_save(x)))


def test_weight_grad_32_bit_gradient_keeps_its_bits(ops):
    """One token with x = 1: dw is dy itself, over the whole range of fp32."""
    g = gen(32)
    n = 512
    dy = randn(g, 1, n) * torch.exp2(torch.randint(-100, 100, (1, n), generator=g, device="cuda").float())
    dy[0, 0], dy[0, 1], dy[0, 2] = torch.finfo(F32).max, -torch.finfo(F32).max, 0.0
    a = ops.act_save(torch.ones(1, 128, device="cuda"))
    dw = ops.weight_grad(dy, a)
    assert torch.equal(dw, dy.view(n, 1).expand(n, 128))


@pytest.mark.parametrize("dt", [BF, F32])
def test_weight_grad_non_finite(ops, dt):
    """A block that held a NaN reaches its columns only, a NaN or an infinity of dy its row only."""
    x = torch.ones(200, 384, dtype=dt, device="cuda")
    x[150, 140] = math.inf
    dy = torch.ones(200, 70, dtype=dt, device="cuda")
    dy[199, 33], dy[3, 40] = math.nan, -math.inf
    dw = ops.weight_grad(dy, ops.act_save(x))
    bad = torch.zeros(70, 384, dtype=torch.bool, device="cuda")
    bad[:, 128:256] = True
    bad[33] = True
    assert torch.equal(torch.isnan(dw), bad)
    assert (dw[40][~bad[40]] == -math.inf).all()
    bad[40] = True
    assert (dw[~bad] == 200).all()


def test_weight_grad_nothing(ops):
    a = ops.Act.empty(0, 100, "cuda")
    dy = torch.empty(0, 30, dtype=BF, device="cuda")
    assert (ops.weight_grad(dy, a) == 0).all()
    base = torch.ones(30, 100, device="cuda")
    ops.weight_grad(dy, a, grad=base, accumulate=True)
    assert (base == 1).all()


def test_weight_grad_is_the_derivative(ops):
    """Central differences of sum(dy * (x W^T)) in 64 bits, x as the checkpoint has it."""
    g = gen(33)
    t, n, k = 9, 4, 6
    a = ops.act_save(randn(g, t, k))
    x, dy = values(a.q, a.e)[:, :k], randn(g, t, n)
    dw = ops.weight_grad(dy, a)
    w = randn(g, n, k).double()
    h = 1e-3
    for i in range(n):
        for j in range(k):
            up, down = w.clone(), w.clone()
            up[i, j] += h
            down[i, j] -= h
            slope = float((dy.double() * (x @ up.t() - x @ down.t())).sum()) / (2 * h)
            assert abs(slope - float(dw[i, j])) < 1e-4


# --- streams and refusals --------------------------------------------------------------------------------------

def test_ops_on_another_stream_and_in_a_graph(ops):
    g = gen(41)
    t, v, d, n = 300, 500, 256, 192
    table, ids = randn(g, v, d, dtype=BF), torch.randint(0, v, (t,), generator=g, device="cuda")
    w, dy, dz = torch.ones(d, dtype=BF, device="cuda"), randn(g, t, d, dtype=BF), randn(g, t, n, dtype=BF)

    def step():
        x = ops.embed(table, ids, scale=2.0)
        y, mean, rstd, keep = ops.norm(x, w, kind="rms", keep=True)
        dw = ops.weight_grad(dz, ops.act_save(y))
        dx, dg, _ = ops.norm_grad(dy, keep, w, mean, rstd)
        return y, dw, dg, ops.embed_grad(dx, ids, v, scale=2.0)
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            held = step()
    for o in held:
        o.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_ops_refuse(ops):
    from paper_2609_27193_gb300 import LCError, _abi
    x = torch.zeros(8, 64, dtype=BF, device="cuda")
    w = torch.ones(64, dtype=BF, device="cuda")
    ids = torch.zeros(8, dtype=torch.int64, device="cuda")
    a = ops.act_save(x)
    _, mean, rstd = ops.norm(x, w)
    with pytest.raises(TypeError):
        ops.norm(x.half(), w)
    with pytest.raises(TypeError):
        ops.embed(x, ids.float())
    with pytest.raises(ValueError):
        ops.embed(x.t(), ids)
    with pytest.raises(ValueError):
        ops.embed(x, ids.cpu())
    with pytest.raises(ValueError):
        ops.norm(x, w[:32])
    with pytest.raises(ValueError):
        ops.embed_grad(x, ids[:4], 10)
    with pytest.raises(ValueError):
        ops.embed_grad(x, ids, 10, accumulate=True)
    with pytest.raises(ValueError):
        ops.weight_grad(x[:4], a)
    with pytest.raises(ValueError):
        ops.norm_grad(x, x, w, mean, rstd[:4])
    with pytest.raises(KeyError):
        ops.norm(x, w, kind="batch")
    with pytest.raises(LCError) as err:
        ops.norm(x, w, out=x)
    assert err.value.status == _abi.LC_ERR_INVALID_ARG and "overlaps" in str(err.value)
    with pytest.raises(LCError, match="overlaps"):
        ops.norm_grad(x, x.clone(), w, mean, rstd, dx=x)
    with pytest.raises(LCError, match="overlaps"):
        ops.embed(x, ids, out=x)
    with pytest.raises(LCError, match="LC_NORM_MAX_DIM"):
        ops.norm(torch.zeros(1, 16385, device="cuda"), torch.zeros(16385, device="cuda"))
    with pytest.raises(LCError, match="eps"):
        ops.norm(x, w, eps=-1.0)
    with pytest.raises(LCError, match="stride"):
        ops.embed(x, ids, out=torch.zeros(1, 64, dtype=BF, device="cuda").expand(8, 64))
    with pytest.raises(LCError, match="checkpoint"):
        ops.weight_grad(x, ops.Act(torch.zeros(8 * 129, dtype=torch.int8, device="cuda").view(8, 129)[:, 1:], a.e, 64))
    # interleaved columns of one buffer are two arrays
    both = torch.zeros(8, 128, dtype=BF, device="cuda")
    ops.norm(both[:, :64], w, out=both[:, 64:])
    lib = _abi.load()
    r = _abi.lc_rows(x.data_ptr(), 64, _abi.LC_BF16, 0)
    host = torch.zeros(8, 64, dtype=BF)
    h = _abi.lc_rows(host.data_ptr(), 64, _abi.LC_BF16, 0)
    assert lib.lc_embed(0, None, h, 8, 64, ids.data_ptr(), _abi.LC_I64, 8, 1.0, r) == _abi.LC_ERR_INVALID_ARG
    assert b"not device memory" in lib.lc_last_error()
    many = torch.zeros(100, dtype=torch.int64, device="cuda")
    long = torch.zeros(100, 64, dtype=BF, device="cuda")
    need = lib.lc_embed_grad_workspace(100, 10, 64)
    g = torch.zeros(10, 64, device="cuda")
    rg = _abi.lc_rows(g.data_ptr(), 64, _abi.LC_F32, 0)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    rl = _abi.lc_rows(long.data_ptr(), 64, _abi.LC_BF16, 0)
    args = (0, None, rl, many.data_ptr(), _abi.LC_I64, 100, 1.0, -1, rg, 10, 64, 0)
    assert lib.lc_embed_grad(*args, ws.data_ptr(), need - 1) == _abi.LC_ERR_CAPACITY
    assert lib.lc_embed_grad(*args, ws.data_ptr() + 8, need) == _abi.LC_ERR_INVALID_ARG
    assert lib.lc_embed_grad(*args, None, need) == _abi.LC_ERR_INVALID_ARG
    assert lib.lc_embed(99, None, r, 8, 64, ids.data_ptr(), _abi.LC_I64, 8, 1.0, r) == _abi.LC_ERR_INVALID_ARG
    torch.cuda.synchronize()
