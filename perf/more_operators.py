"""More operators of a training step, as cases that can be timed and compared: what lies between two linear layers, and
what a matrix's gradient goes through before it updates the matrix.

  add_norm       a branch's output is added to the residual stream, and the sum's root-mean-square norm is the next
                 branch's input; on request the sum and the norm's output are also kept in 8 bits (blocks of 128 values of
                 one token share a power of two, the values are whole numbers of [-127, 127])
  add_norm_grad  the gradient of both addends and of the norm's weight, from the sum or from its 8-bit checkpoint
  orthogonalize  an update of a weight matrix, or of a batch of them, made nearly orthogonal by Newton-Schulz products,
                 X <- a X + (b A + c A^2) X with A = X X^T, five times from the update over its Frobenius norm; on request
                 the update comes out of a momentum buffer that the same call moves

Widths, projections and types are those of the workloads' layouts (d 256, 768, 2048, 4096; ffn 1024, 8192, 14336; key
projections of 512 and 1024 rows), token counts go from one to eight sequences of 2048.
"""
import math

import torch

own = False

BLOCK = 128                    # values that share an exponent in a checkpoint
EPS = 1e-5
TINY = 1e-7                    # added to an update's norm
COEF = (3.4445, -4.7750, 2.0315)
STEPS, BETA = 5, 0.95
BF16, F32 = "bf16", "f32"
_DT = {BF16: torch.bfloat16, F32: torch.float32}


def listed():
    return [
        # a single sequence's last few tokens through the smallest model: the call's latency is all of it
        dict(name="add_norm 64x256", path="add_norm", tokens=64, dim=256, dtype=BF16, stream=BF16, keep=False, out8=False),
        # an odd number of tokens of the 1.2 G model, the residual stream in 32 bits and kept in 8 for the backward
        dict(name="add_norm 4099x2048 f32 keep", path="add_norm", tokens=4099, dim=2048, dtype=BF16, stream=F32, keep=True,
             out8=False),
        # eight sequences of the largest layout; the norm's output is also kept in 8 bits for the next layer's weight gradient
        dict(name="add_norm 16Kx4096 out8", path="add_norm", tokens=16384, dim=4096, dtype=BF16, stream=BF16, keep=False,
             out8=True),
        # one sequence less a token at a width between the layouts', backward from the sum itself
        dict(name="add_norm_grad 2047x768", path="add_norm_grad", tokens=2047, dim=768, dtype=BF16, stream=BF16, kept=False),
        # four sequences of the 1.2 G model, the stream's gradient in 32 bits
        dict(name="add_norm_grad 8191x2048 f32", path="add_norm_grad", tokens=8191, dim=2048, dtype=BF16, stream=F32,
             kept=False),
        # eight sequences of the largest layout, backward from the checkpoint
        dict(name="add_norm_grad 16Kx4096 kept", path="add_norm_grad", tokens=16384, dim=4096, dtype=BF16, stream=BF16,
             kept=True),
        # a projection of the smallest model: fifteen products one after the other that each take next to nothing
        dict(name="orthogonalize 256x256", path="orthogonalize", batch=1, rows=256, cols=256, dtype=F32, momentum=False),
        # the up and gate projections of all four blocks of the smallest model at once, through their momentum
        dict(name="orthogonalize 8x1024x256", path="orthogonalize", batch=8, rows=1024, cols=256, dtype=F32, momentum=True),
        # a matrix that fits no tile
        dict(name="orthogonalize 515x1023", path="orthogonalize", batch=1, rows=515, cols=1023, dtype=BF16, momentum=False),
        # a key projection of the largest layout
        dict(name="orthogonalize 1024x4096", path="orthogonalize", batch=1, rows=1024, cols=4096, dtype=BF16, momentum=False),
        # the up projection of the 1.2 G model (more rows than columns), through its momentum
        dict(name="orthogonalize 8192x2048", path="orthogonalize", batch=1, rows=8192, cols=2048, dtype=F32, momentum=True),
        # the down projection of the largest layout
        dict(name="orthogonalize 4096x14336", path="orthogonalize", batch=1, rows=4096, cols=14336, dtype=F32,
             momentum=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width over [lo, hi]: half of them whole blocks of 128, a quarter multiples of 8, a quarter anything."""
    n = _log(rng, lo, hi)
    to = rng.choice((BLOCK, BLOCK, 8, 1))
    return min(hi, max(to, -(-n // to) * to))


def draw(rng):
    path = rng.choice(("add_norm", "add_norm_grad", "orthogonalize"))
    if path == "orthogonalize":
        rows, cols = _width(rng, 16, 4096), _width(rng, 16, 14336)
        if rng.random() < 0.5:
            rows, cols = cols, rows
        batch = min(_log(rng, 1, 16) if rng.random() < 0.5 else 1, max(1, (1 << 24) // (rows * cols)))
        return dict(path=path, batch=batch, rows=rows, cols=cols, dtype=rng.choice((BF16, F32)), momentum=rng.random() < 0.5)
    dtype, stream = rng.choice(((BF16, BF16), (BF16, BF16), (BF16, F32), (F32, F32)))
    c = dict(path=path, tokens=_log(rng, 1, 16384), dim=_width(rng, 64, 4096), dtype=dtype, stream=stream)
    if path == "add_norm":
        c.update(keep=rng.random() < 0.5, out8=rng.random() < 0.5)
    else:
        c.update(kept=rng.random() < 0.5)
    return c


# --- inputs ---------------------------------------------------------------------------------------------------

def _activation(g, t, d, dtype, spread=1.0):
    """Activations of a residual stream: normal, with a few features that are much larger than the others."""
    x = torch.randn(t, d, generator=g, device="cuda")
    size = torch.exp(0.5 * torch.randn(d, generator=g, device="cuda"))
    return (x * size * spread).to(_DT[dtype])


def _gradient(g, b, m, n, dtype):
    """Gradients of weight matrices: a few directions of many tokens over a floor of noise, with rows and columns of
    different sizes."""
    r = max(1, min(m, n) // 4)
    u = torch.randn(b, m, r, generator=g, device="cuda")
    v = torch.randn(b, r, n, generator=g, device="cuda")
    size = 1.0 / torch.arange(1, r + 1, device="cuda")
    x = torch.bmm(u * size.sqrt(), v) + 0.5 * torch.randn(b, m, n, generator=g, device="cuda")
    x *= torch.exp(0.3 * torch.randn(b, m, 1, generator=g, device="cuda"))
    x *= torch.exp(0.3 * torch.randn(b, 1, n, generator=g, device="cuda"))
    return (1e-3 * x).to(_DT[dtype])


def _pow2(e):
    """2^e for whole numbers e in [-126, 127], from the bits of an fp32 number."""
    return (e.int() + 127 << 23).view(torch.float32)


def _quantize(x):
    """(q, e): the checkpoint of x in its public layout: int8 [tokens, blocks * 128] and int8 [tokens, blocks]."""
    t, d = x.shape
    nb = -(-d // BLOCK)
    v = torch.zeros(t, nb * BLOCK, device="cuda")
    v[:, :d] = x
    v = v.view(t, nb, BLOCK)
    m, k = torch.frexp(v.abs().amax(2))
    e = torch.where(m <= 127 / 128, k - 7, k - 6).clamp_(min=-126)
    e = torch.where(m == 0, -126, e)
    q = torch.round(v * _pow2(-e)[:, :, None]).to(torch.int8)
    return q.view(t, nb * BLOCK), e.to(torch.int8)


def _values(q, e, d, dtype=torch.float32):
    t, nb = e.shape
    v = q.view(t, nb, BLOCK).to(dtype) * _pow2(e).to(dtype)[:, :, None]
    return v.reshape(t, nb * BLOCK)[:, :d]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=c)
    if c["path"] == "orthogonalize":
        shape = (c["batch"], c["rows"], c["cols"])
        s["update"] = _gradient(g, *shape, c["dtype"])
        s["momentum"] = _gradient(g, *shape, F32) if c["momentum"] else None
        return s
    t, d = c["tokens"], c["dim"]
    s["weight"] = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(_DT[c["dtype"]])
    if c["path"] == "add_norm":
        s["x"] = _activation(g, t, d, c["dtype"], 0.3)
        s["residual"] = _activation(g, t, d, c["stream"])
        return s
    total = _activation(g, t, d, c["stream"])
    if c["kept"]:
        s["q"], s["e"] = _quantize(total)
        total = _values(s["q"], s["e"], d)
    else:
        s["sum"] = total
    s["rstd"] = torch.rsqrt(total.float().square().mean(1) + EPS)
    s["dy"] = _activation(g, t, d, c["dtype"], 1e-3)
    s["dsum"] = _activation(g, t, d, c["stream"], 1e-3)
    return s


# --- the operators --------------------------------------------------------------------------------------------

def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2609_27193_gb300 import ops
    c = s["case"]
    if c["path"] == "add_norm":
        total, y, rstd, *kept = ops.add_norm(s["x"], s["residual"], s["weight"], eps=EPS, keep=c["keep"] or None,
                                             out8=c["out8"] or None)
        out = dict(sum=total, y=y, rstd=rstd)
        # what is kept in 8 bits is returned as its values
        if c["keep"]:
            out["kept"] = ops.act_load(kept[0])
        if c["out8"]:
            out["y8"] = ops.act_load(kept[-1])
        return out
    if c["path"] == "add_norm_grad":
        total = ops.Act(s["q"], s["e"], c["dim"]) if c["kept"] else s["sum"]
        dx, dw = ops.add_norm_grad(s["dy"], s["dsum"], total, s["weight"], s["rstd"])
        return dict(dx=dx, dweight=dw)
    out = ops.orthogonalize(s["update"], momentum=s["momentum"], beta=BETA, steps=STEPS, coefficients=COEF, eps=TINY)
    return dict(out=out, momentum=s["momentum"])


def _plain(s):
    c = s["case"]
    if c["path"] == "add_norm":
        total = s["x"].float() + s["residual"].float()
        rstd = torch.rsqrt((total * total).mean(1) + EPS)
        y = total * rstd[:, None] * s["weight"].float()
        out = dict(sum=total.to(_DT[c["stream"]]), y=y.to(_DT[c["dtype"]]), rstd=rstd)
        if c["keep"]:
            out["kept"] = _values(*_quantize(total), c["dim"]).to(torch.bfloat16)
        if c["out8"]:
            out["y8"] = _values(*_quantize(y), c["dim"]).to(torch.bfloat16)
        return out
    if c["path"] == "add_norm_grad":
        h = _values(s["q"], s["e"], c["dim"]) if c["kept"] else s["sum"].float()
        h = h * s["rstd"][:, None]
        dy = s["dy"].float()
        a = dy * s["weight"].float()
        dx = s["dsum"].float() + (a - h * (a * h).mean(1, keepdim=True)) * s["rstd"][:, None]
        return dict(dx=dx.to(_DT[c["stream"]]), dweight=(dy * h).sum(0))
    x = s["update"].float()
    m = s["momentum"]
    if m is not None:
        m += (1 - BETA) * (x - m)          # the buffer moves towards the gradient
        x = x + BETA * (m - x)             # and the update looks one step ahead
    a, b, k = COEF
    turned = c["rows"] > c["cols"]
    if turned:
        x = x.transpose(1, 2)
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + TINY)
    for _ in range(STEPS):
        p = torch.matmul(x, x.transpose(1, 2))
        p = b * p + k * torch.matmul(p, p)
        x = a * x + torch.matmul(p, x)
    if turned:
        x = x.transpose(1, 2)
    return dict(out=x.to(torch.bfloat16), momentum=m)


# --- the same in 64 bits, from the definitions ----------------------------------------------------------------

def _exact8(x):
    """The definition of a checkpoint, block by block on whole columns: the smallest power of two (from 2^-126) with which
    127 steps reach the block's largest value, and the nearest of those steps, halves to the even one."""
    out = torch.empty_like(x)
    for b in range(0, x.shape[1], BLOCK):
        v = x[:, b:b + BLOCK]
        most = v.abs().amax(1, keepdim=True)
        step = torch.exp2(torch.ceil(torch.log2(most.clamp_min(2.0 ** -140) / 127)))
        step = torch.where(step * 63.5 >= most, step / 2, step)    # log2's rounding
        step = torch.where(step * 127 < most, step * 2, step).clamp_min(2.0 ** -126)
        out[:, b:b + BLOCK] = torch.round(v / step) * step
    return out


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    if c["path"] == "add_norm":
        total = s["x"].double() + s["residual"].double()
        rstd = 1 / (total.pow(2).sum(1) / c["dim"] + EPS).sqrt()
        y = torch.einsum("td,t,d->td", total, rstd, s["weight"].double())
        out = dict(sum=total, y=y, rstd=rstd)
        if c["keep"]:
            out["kept"] = _exact8(total)
        if c["out8"]:
            out["y8"] = _exact8(y)
        return out
    if c["path"] == "add_norm_grad":
        h = _values(s["q"], s["e"], c["dim"], torch.float64) if c["kept"] else s["sum"].double()
        rstd, dy = s["rstd"].double(), s["dy"].double()
        h = torch.einsum("td,t->td", h, rstd)
        a = dy * s["weight"].double()
        along = torch.einsum("td,td->t", a, h) / c["dim"]
        dx = s["dsum"].double() + torch.einsum("td,t->td", a, rstd) - torch.einsum("td,t->td", h, along * rstd)
        return dict(dx=dx, dweight=torch.einsum("td,td->d", dy, h))
    # every step multiplies from the left by a polynomial of A = X X^T, and all of these commute: the steps on the Gram
    # matrix alone, their product applied to the update once
    x, m = s["update"].double(), None
    if s["momentum"] is not None:
        m = BETA * s["momentum"].double() + (1 - BETA) * x
        x = (1 - BETA) * x + BETA * m
    turned = c["rows"] > c["cols"]
    outs = []
    for v in x:
        v = v.t() if turned else v
        v = v / (torch.linalg.norm(v) + TINY)
        gram = v @ v.t()
        eye = torch.eye(gram.shape[0], dtype=torch.float64, device="cuda")
        every = eye
        for _ in range(STEPS):
            step = COEF[0] * eye + gram @ (COEF[1] * eye + COEF[2] * gram)
            gram = step @ gram @ step
            every = step @ every
        v = every @ v
        outs.append(v.t() if turned else v)
    return dict(out=torch.stack(outs), momentum=m)


# --- what a pass cannot do without ----------------------------------------------------------------------------

def work(case):
    c = dict(case)
    if c["path"] == "orthogonalize":
        # A and A^2 are symmetric: half of their products are needed
        e = 2 if c["dtype"] == BF16 else 4
        m, n = sorted((c["rows"], c["cols"]))
        every = c["batch"] * m * n
        return dict(bytes=every * (e + 2 + (8 if c["momentum"] else 0)), flops=c["batch"] * STEPS * m * (m * n + m * m + 2 * m * n))
    t, d = c["tokens"], c["dim"]
    e = 2 if c["dtype"] == BF16 else 4
    r = 2 if c["stream"] == BF16 else 4
    nb = -(-d // BLOCK)
    act = t * nb * (BLOCK + 1)                      # bytes of a checkpoint
    if c["path"] == "add_norm":
        # x, residual, sum, y; a checkpoint is written, read back and its values written
        return dict(bytes=2 * (e + r) * t * d + 4 * t + e * d + (c["keep"] + c["out8"]) * (2 * act + 2 * t * d), flops=7 * t * d)
    return dict(bytes=(e + 2 * r) * t * d + (act if c["kept"] else r * t * d) + 4 * t + e * d + 4 * d, flops=11 * t * d)
