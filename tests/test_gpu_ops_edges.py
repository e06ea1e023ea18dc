"""The operators at the sizes where one shape of a kernel ends and the next begins, with outputs that start as NaN
and sums that fp32 holds exactly."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import (BF, F32, IDS, SUMS, U, gen, make_ids, norm_grad_ref, norm_ref, quantize, randn, values,  # noqa: E402
                                within)


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import ops
    return ops


def whole(g, *shape, dtype=F32, most=3):
    """Whole numbers of [-most, most]: a sum of up to 2^24 / most of them has no rounding in fp32."""
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").to(dtype)


# --- norm ------------------------------------------------------------------------------------------------------

# widths at which a group of threads or its vectors change, one 16-byte vector to either side
EDGES = [(d + s, dt) for d in (256, 512, 768, 1024, 2048, 4096, 8192) for dt, v in ((F32, 4), (BF, 8)) for s in (-v, 0, v)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("t", [5, 311])
@pytest.mark.parametrize("d,dt", EDGES)
def test_norm_between_its_shapes(ops, kind, t, d, dt):
    """Both directions, directly and through the rings: every column is written and counted."""
    g = gen(t * d)
    x = (randn(g, t, d) + (2.0 if kind == "layer" else 0.0)).to(dt)
    x[:, -4:] *= 4                                        # the last columns weigh in the statistics
    w = 1 + randn(g, d, dtype=dt, spread=0.2)
    b = randn(g, d, dtype=dt) if kind == "layer" else None
    out = torch.full((t, d), math.nan, dtype=dt, device="cuda")
    keep = ops.Act.empty(t, d, "cuda")
    keep.q.fill_(55)
    keep.e.fill_(55)
    y, mean, rstd = ops.norm(x, w, b, kind=kind, out=out, keep=keep)
    ref, rmean, rrstd, xhat = norm_ref(x, w, b, kind, 1e-5)
    a = x.double().abs().mean(1)
    if mean is not None:
        within(mean, rmean, SUMS * U * a, "mean")
    within(rstd, rrstd, (SUMS + 4) * U * rrstd, "rstd")
    room = ((SUMS + 8) * U * xhat.abs() + (SUMS + 8) * U * (a * rrstd)[:, None]) * w.double().abs()
    within(y, ref, room + (4 * U * b.double().abs() if b is not None else 0), "y")
    q, e, _ = quantize(x)
    assert torch.equal(keep.q, q) and torch.equal(keep.e, e)
    dy = whole(g, t, d, dtype=dt)
    for kept in (False, True):
        seen = values(keep.q, keep.e)[:, :d] if kept else x
        dx = torch.full((t, d), math.nan, dtype=dt, device="cuda")
        # without a bias the root-mean-square norm has a form of its own
        for bias in (True, False):
            dx.fill_(math.nan)
            dw = torch.full((d,), math.nan, device="cuda")
            db = torch.full((d,), math.nan, device="cuda") if bias else None
            ops.norm_grad(dy, keep if kept else x, w, mean, rstd, dx=dx, dweight=dw, dbias=db)
            rdx, room, rdw, wroom, rdb, _ = norm_grad_ref(dy, seen, w, mean, rstd)
            within(dx, rdx, room, "dx")
            within(dw, rdw, wroom, "dweight")
            assert db is None or torch.equal(db.double(), rdb)


# --- weight gradient -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dt,gt", [(BF, F32), (BF, BF), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("t,n,k", [(64, 2560, 2816), (1100, 2500, 2900), (8192, 1030, 5200), (65, 128, 20500), (2049, 4099, 1300)])
def test_weight_grad_of_several_tiles_a_pair(ops, dt, gt, t, n, k):
    """More output tiles than the device holds pairs of CTAs: what the rings and accumulators carry from a tile to the
    next, ends inside a chain, outputs written while the next tile's products run.  Whole numbers, so that every order of
    adding them gives the same sums: 3 * 3 * 8192 and what is added to stay below 2^24."""
    g = gen(t + n)
    dy, x = whole(g, t, n, dtype=dt), whole(g, t, k, dtype=dt)
    x[:, ::128] = 64.0                                    # with steps of 1 a value is a whole number of them
    a = ops.act_save(x)
    assert torch.equal(ops.act_load(a, dtype=dt), x)
    ref = dy.double().t() @ x.double()
    out = torch.full((n, k), math.nan, dtype=gt, device="cuda")
    for _ in range(3):
        ops.weight_grad(dy, a, grad=out)
        assert torch.equal(out, ref.to(gt))
    base = whole(g, n, k, dtype=gt, most=100)
    out.copy_(base)
    ops.weight_grad(dy, a, grad=out, accumulate=True)
    assert torch.equal(out, (ref + base.double()).to(gt))


# --- scratch in graphs -----------------------------------------------------------------------------------------

def graph_inputs(seed, t=700, v=300, d=256, n=192):
    g = gen(seed)
    return dict(v=v, ids=torch.randint(0, v, (t,), generator=g, device="cuda"), x=randn(g, t, d, dtype=BF),
                w=1 + randn(g, d, dtype=BF, spread=0.2), dy=randn(g, t, d, dtype=BF), dz=randn(g, t, n))


def graph_step(ops, s):
    """Every call that takes scratch."""
    y, mean, rstd = ops.norm(s["x"], s["w"])
    dx, dw, db = ops.norm_grad(s["dy"], s["x"], s["w"], mean, rstd, bias=True)
    return [y, dx, dw, db, ops.weight_grad(s["dz"], ops.act_save(s["x"])), ops.embed_grad(dx, s["ids"], s["v"], dtype=F32)]


def captured(ops, s, stream):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = graph_step(ops, s)
    return graph, out


def test_a_graph_keeps_its_scratch(ops):
    """After a larger call on the stream that the graph was captured on, replays write to nobody else's memory."""
    side = torch.cuda.Stream()
    s = graph_inputs(51)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = graph_step(ops, s)                         # the scratch that there is before the capture
    side.synchronize()
    graph, held = captured(ops, s, side)
    with torch.cuda.stream(side):
        big = graph_step(ops, graph_inputs(52, t=9000, v=5000, d=1024, n=512))
        # whatever was given back is handed out again
        fills = [torch.full((1 << k,), 0x5a, dtype=torch.uint8, device="cuda") for k in range(12, 25) for _ in range(3)]
    side.synchronize()
    for o in held:
        o.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, want))
    assert all(bool((f == 0x5a).all()) for f in fills)
    assert all(bool(torch.isfinite(b).all()) for b in big)


def test_graphs_of_one_stream_on_two(ops):
    """Captured on one stream, replayed side by side."""
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    inputs = [graph_inputs(53, t=20000), graph_inputs(54, t=20000)]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        wants = [graph_step(ops, s) for s in inputs]
    side.synchronize()
    graphs = [captured(ops, s, side) for s in inputs]
    for _, held in graphs:
        for o in held:
            o.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for (graph, _), stream in zip(graphs, (side, other)):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for (_, held), want in zip(graphs, wants):
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_large_scratch_is_given_back(ops):
    """A 32-bit dy is staged as three bf16 parts: 100 MB here, none of it held after the call."""
    g = gen(55)
    t, n = 8192, 2048
    dy, a = whole(g, t, n), ops.act_save(whole(g, t, 128))
    ref = dy.double().t() @ ops.act_load(a, dtype=F32).double()
    ops.weight_grad(dy[:100], ops.act_save(whole(g, 100, 128)))
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    dw = ops.weight_grad(dy, a)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - before <= dw.numel() * 4 + (32 << 20)
    assert torch.equal(dw, ref.float())


# --- the sums over tokens, exactly -----------------------------------------------------------------------------

@pytest.mark.parametrize("how", IDS)
@pytest.mark.parametrize("t,v,d,dt,gt", [
    (64, 70, 2048, BF, F32), (65, 70, 200, F32, F32), (777, 513, 256, F32, BF), (2049, 131072, 24, F32, F32),
    (16381, 32000, 768, BF, BF), (20011, 40, 1030, BF, F32), (20011, 40, 1031, BF, F32), (65536, 128256, 8, BF, F32),
    (65537, 3000, 40, BF, F32), (70001, 300, 8, BF, F32), (140000, 70000, 16, BF, F32), (300000, 5, 129, F32, F32)])
def test_embed_grad_of_whole_numbers(ops, how, t, v, d, dt, gt):
    """Sums that fp32 holds exactly (at most 3 * 300000): a token that is lost, doubled or in another row shows,
    also in a row that all tokens share."""
    g = gen(t + d)
    dy = whole(g, t, d, dtype=dt)
    ids = make_ids(g, t, v, how)
    ref = torch.zeros(v, d, dtype=torch.float64, device="cuda")
    keep = ids >= 0
    ref.index_add_(0, ids[keep], dy[keep].double())
    grad = torch.full((v, d), math.nan, dtype=gt, device="cuda")
    ops.embed_grad(dy, ids, grad=grad)
    assert torch.equal(grad, ref.to(gt))
    base = whole(g, v, d, dtype=gt, most=100)
    grad = base.clone()
    ops.embed_grad(dy, ids, grad=grad, accumulate=True)
    assert torch.equal(grad, (ref + base.double()).to(gt))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("t,d", [(5003, 384), (16384, 256), (9000, 1000), (4000, 4096), (3001, 4095), (40000, 24), (700, 16384)])
def test_norm_bias_gradient_of_whole_numbers(ops, dt, t, d):
    """dbias exactly, of rows of their own and of one row that all share (stride 0)."""
    g = gen(t + d)
    x, w = randn(g, t, d, dtype=dt), torch.ones(d, dtype=dt, device="cuda")
    _, mean, rstd, act = ops.norm(x, w, keep=True)
    for dy in (whole(g, t, d, dtype=dt), whole(g, 1, d, dtype=dt).expand(t, d)):
        for seen in (x, act):
            _, _, db = ops.norm_grad(dy, seen, w, mean, rstd, bias=True)
            assert torch.equal(db.double(), dy.double().sum(0))


@pytest.mark.parametrize("t", [3000, 70000])
def test_embed_grad_of_a_vocabulary_of_28_bits(ops, t):
    """Four digits to sort by, in shared memory and beyond it."""
    g = gen(t)
    v = 2 ** 27 + 5
    ids = torch.randint(0, v, (t,), generator=g, device="cuda")
    ids[t // 2:] = ids[:t - t // 2]                       # every id at least twice
    ids[7], ids[8] = v - 1, 2 ** 27
    dy = whole(g, t, 1)
    grad = ops.embed_grad(dy, ids, v)
    ref = torch.zeros(v, 1, device="cuda").index_add_(0, ids, dy)
    assert torch.equal(grad, ref)


@pytest.mark.parametrize("dt", [BF, F32])
def test_rows_far_apart(ops, dt):
    """Row offsets beyond 32 bits, in elements, for every call."""
    g = gen(71)
    t, d, n = 3, 1024, 256
    far = 2 ** 31 + 64
    buf = torch.empty(2 * far + 4096, dtype=dt, device="cuda")
    out = torch.empty(2 * far + 4096, dtype=dt, device="cuda")
    q8 = torch.zeros(4 * far + 4096, dtype=torch.int8, device="cuda")

    def put(x):
        v = buf.as_strided(x.shape, (far, 1))
        v.copy_(x)
        return v

    def room(*shape):
        return out.as_strided(shape, (far, 1))
    x, dy, w = randn(g, t, d, dtype=dt), randn(g, t, d, dtype=dt), 1 + randn(g, d, dtype=dt, spread=0.2)
    y, mean, rstd, act = ops.norm(x, w, keep=True)
    kept = ops.Act(q8.as_strided((t, d), (2 * far, 1)), q8[2048:].as_strided((t, d // 128), (2 * far, 1)), d)
    got = ops.norm(put(x), w, out=room(t, d), keep=kept)
    assert torch.equal(got[0], y) and torch.equal(got[1], mean) and torch.equal(got[2], rstd)
    assert torch.equal(kept.q, act.q) and torch.equal(kept.e, act.e)
    assert torch.equal(ops.act_load(kept, out=room(t, d)), ops.act_load(act, dtype=dt))
    kept.q.zero_()
    ops.act_save(put(x), kept)
    assert torch.equal(kept.q, act.q)
    want = ops.norm_grad(dy, x, w, mean, rstd, bias=True)
    for a, b in zip(ops.norm_grad(put(dy), x, w, mean, rstd, bias=True, dx=room(t, d)), want):
        assert torch.equal(a, b)
    want = ops.norm_grad(dy, act, w, mean, rstd, bias=True)
    for a, b in zip(ops.norm_grad(put(dy), kept, w, mean, rstd, bias=True), want):
        assert torch.equal(a, b)
    dz = randn(g, t, n, dtype=dt)
    assert torch.equal(ops.weight_grad(put(dz), kept), ops.weight_grad(dz, act))
    dz = whole(g, t, 3, dtype=dt)                         # three rows of the output, far apart
    assert torch.equal(ops.weight_grad(dz, act, grad=room(3, d)), ops.weight_grad(dz, act, dtype=dt))
    ids = torch.tensor([2, 0, 2], device="cuda")
    assert torch.equal(ops.embed_grad(put(dy), ids, grad=room(3, d)), ops.embed_grad(dy, ids, 3))
    many = torch.arange(300, device="cuda") % 3
    rows = whole(g, 300, d, dtype=dt)
    assert torch.equal(ops.embed_grad(rows, many, grad=room(3, d)), ops.embed_grad(rows, many, 3))
