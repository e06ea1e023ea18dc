"""The operators of a training step that feed the fused optimizer step, as cases that can be timed and compared.

The library keeps weights, snapshot, moments and gradients of a model on one GPU.  What lies between two optimizer
steps and meets those arrays directly is measured here, each direction by itself:

  embed       rows of the embedding table for a batch of token ids, times a scale
  embed_grad  the table's gradient: for every row the sum of its tokens' gradients, rows without a token zero (the
              optimizer step reads the whole gradient)
  norm        layer norm or root-mean-square norm of every token's vector, with the statistics the backward reads
  norm_grad   its input's gradient and the gradients of weight and bias, from the input itself or from its 8-bit
              checkpoint
  save        an activation into an 8-bit checkpoint and back out of it: blocks of 128 values of one token share a
              power of two, the values are whole numbers of [-127, 127]
  weight_grad the gradient of a linear layer's weight, dW = dY^T X, with X read from its 8-bit checkpoint

Widths, vocabularies and types are those of the workloads' layouts (d 256, 768, 2048, 4096; ffn 1024, 8192, 14336;
vocabularies 8000, 32000, 128256), token counts go from one to eight sequences of 2048.  Ids are distributed like
words (a few very frequent ones, a long tail), every sixteenth position is masked (id -1) in the gradient's cases.
"""
import math

import torch

own = False

BLOCK = 128                    # values that share an exponent in a checkpoint
EPS = 1e-5
BF16, F32 = "bf16", "f32"
_DT = {BF16: torch.bfloat16, F32: torch.float32}


def listed():
    return [
        # the smallest model's lookup for a few sequences' worth of tokens: the call's latency is all of it
        dict(name="embed 512x256", path="embed", tokens=512, dim=256, vocab=8000, dtype=BF16, scale=16.0),
        # eight sequences of the largest layout, rows scaled by sqrt(d)
        dict(name="embed 16Kx4096", path="embed", tokens=16384, dim=4096, vocab=128256, dtype=BF16, scale=64.0),
        # one sequence less a token into the 32-bit gradient of a 1.2 G model's table: most rows have no token
        dict(name="embed_grad 2047x2048 f32", path="embed_grad", tokens=2047, dim=2048, vocab=128256, dtype=BF16,
             grad=F32, scale=1.0),
        # many tokens over a small table, odd count, 16-bit gradient: frequent words have thousands of tokens
        dict(name="embed_grad 16381x768", path="embed_grad", tokens=16381, dim=768, vocab=32000, dtype=BF16,
             grad=BF16, scale=27.5),
        # layer norm of the smallest model in 32 bits
        dict(name="norm 512x256 f32", path="norm", tokens=512, dim=256, dtype=F32, kind="layer"),
        # eight sequences of the largest layout through a root-mean-square norm
        dict(name="norm 16Kx4096 rms", path="norm", tokens=16384, dim=4096, dtype=BF16, kind="rms"),
        # an odd number of tokens of the 1.2 G model, backward from the input itself
        dict(name="norm_grad 4099x2048", path="norm_grad", tokens=4099, dim=2048, dtype=BF16, kind="layer", kept=False),
        # eight sequences of the largest layout, backward from the checkpoint
        dict(name="norm_grad 16Kx4096 kept", path="norm_grad", tokens=16384, dim=4096, dtype=BF16, kind="rms", kept=True),
        # one sequence of the widest activation there is (ffn), into a checkpoint and back
        dict(name="save 2047x14336", path="save", tokens=2047, dim=14336, dtype=BF16),
        # the smallest model's up projection: few output tiles, so the tokens have to be split
        dict(name="weight_grad 512 256->1024", path="weight_grad", tokens=512, rows=1024, dim=256, dtype=BF16, grad=F32),
        # a key projection of the 1.2 G model whose output gradient is kept in 32 bits
        dict(name="weight_grad 2047 2048->512 f32", path="weight_grad", tokens=2047, rows=512, dim=2048, dtype=F32,
             grad=F32),
        # the down projection of the largest layout over four sequences
        dict(name="weight_grad 8K 14336->4096", path="weight_grad", tokens=8192, rows=4096, dim=14336, dtype=BF16,
             grad=F32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width over [lo, hi]: half of them whole blocks of 128, a quarter multiples of 8, a quarter anything."""
    n = _log(rng, lo, hi)
    to = rng.choice((BLOCK, BLOCK, 8, 1))
    return min(hi, max(to, -(-n // to) * to))


def draw(rng):
    path = rng.choice(("embed", "embed_grad", "norm", "norm_grad", "save", "weight_grad"))
    c = dict(path=path, tokens=_log(rng, 1, 16384), dim=_width(rng, 64, 4096), dtype=rng.choice((BF16, BF16, F32)))
    if path in ("embed", "embed_grad"):
        c.update(vocab=_log(rng, 1000, 128256), scale=rng.choice((1.0, 27.5, 64.0)))
    if path in ("norm", "norm_grad"):
        c.update(kind=rng.choice(("layer", "rms")))
    if path == "norm_grad":
        c.update(kept=rng.random() < 0.5)
    if path == "save":
        c.update(dim=_width(rng, 64, 14336), tokens=min(c["tokens"], 8192))
    if path == "weight_grad":
        c.update(rows=_width(rng, 64, 4096), tokens=min(c["tokens"], 8192), dim=_width(rng, 64, 14336))
    if path in ("embed_grad", "weight_grad"):
        c.update(grad=rng.choice((BF16, F32)))
    return c


# --- inputs ---------------------------------------------------------------------------------------------------

def _activation(g, t, d, dtype, spread=1.0):
    """Activations of a residual stream: normal, with a few features that are much larger than the others."""
    x = torch.randn(t, d, generator=g, device="cuda")
    size = torch.exp(0.5 * torch.randn(d, generator=g, device="cuda"))
    return (x * size * spread).to(_DT[dtype])


def _ids(g, t, vocab, masked):
    """Word-like ids: the k-th most frequent word about 1/k as often, words in no particular order."""
    u = torch.rand(t, generator=g, device="cuda")
    rank = (torch.pow(float(vocab), u) - 1.0).long().clamp_(0, vocab - 1)
    ids = torch.randperm(vocab, generator=g, device="cuda")[rank]
    if masked:
        ids[torch.rand(t, generator=g, device="cuda") < 1 / 16] = -1
    return ids


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
    t, d, path = c["tokens"], c["dim"], c["path"]
    s = dict(case=c)
    if path == "embed":
        s["table"] = (0.02 * torch.randn(c["vocab"], d, generator=g, device="cuda")).to(_DT[c["dtype"]])
        s["ids"] = _ids(g, t, c["vocab"], False)
    elif path == "embed_grad":
        s["dy"] = _activation(g, t, d, c["dtype"], 1e-3)
        s["ids"] = _ids(g, t, c["vocab"], True)
    elif path == "save":
        s["x"] = _activation(g, t, d, c["dtype"])
    elif path == "weight_grad":
        s["q"], s["e"] = _quantize(_activation(g, t, d, c["dtype"]))
        s["dy"] = _activation(g, t, c["rows"], c["dtype"], 1e-3)
    else:
        x = _activation(g, t, d, c["dtype"])
        s["weight"] = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(_DT[c["dtype"]])
        s["bias"] = (0.1 * torch.randn(d, generator=g, device="cuda")).to(_DT[c["dtype"]]) if c["kind"] == "layer" else None
        if path == "norm":
            s["x"] = x
        else:
            s["dy"] = _activation(g, t, d, c["dtype"], 1e-3)
            if c["kept"]:
                s["q"], s["e"] = _quantize(x)
                x = _values(s["q"], s["e"], d)
            else:
                s["x"] = x
            v = x.float()
            s["mean"] = v.mean(1) if c["kind"] == "layer" else None
            if c["kind"] == "layer":
                v = v - s["mean"][:, None]
            s["rstd"] = torch.rsqrt((v * v).mean(1) + EPS)
    return s


# --- the operators --------------------------------------------------------------------------------------------

def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2609_27193_gb300 import ops
    c = s["case"]
    path = c["path"]
    if path == "embed":
        return dict(y=ops.embed(s["table"], s["ids"], scale=c["scale"]))
    if path == "embed_grad":
        return dict(grad=ops.embed_grad(s["dy"], s["ids"], c["vocab"], scale=c["scale"], dtype=_DT[c["grad"]]))
    if path == "norm":
        y, mean, rstd = ops.norm(s["x"], s["weight"], s["bias"], eps=EPS, kind=c["kind"])
        return dict(y=y, mean=mean, rstd=rstd)
    if path == "norm_grad":
        x = ops.Act(s["q"], s["e"], c["dim"]) if c["kept"] else s["x"]
        dx, dw, db = ops.norm_grad(s["dy"], x, s["weight"], s["mean"], s["rstd"], bias=s["bias"] is not None)
        return dict(dx=dx, dweight=dw, dbias=db)
    if path == "save":
        return dict(x=ops.act_load(ops.act_save(s["x"]), dtype=s["x"].dtype))
    return dict(dw=ops.weight_grad(s["dy"], ops.Act(s["q"], s["e"], c["dim"]), dtype=_DT[c["grad"]]))


def _plain(s):
    c = s["case"]
    path, dt = c["path"], _DT[c["dtype"]]
    if path == "embed":
        return dict(y=(s["table"][s["ids"]].float() * c["scale"]).to(dt))
    if path == "embed_grad":
        t = s["ids"].numel()
        # masked positions go to a row behind the table
        row = torch.where(s["ids"] < 0, c["vocab"], s["ids"])
        grad = torch.zeros(c["vocab"] + 1, c["dim"], device="cuda")
        grad.index_add_(0, row, s["dy"].float() * c["scale"])
        return dict(grad=grad[:c["vocab"]].to(_DT[c["grad"]]))
    if path == "norm":
        v = s["x"].float()
        mean = None
        if c["kind"] == "layer":
            mean = v.mean(1)
            v = v - mean[:, None]
        rstd = torch.rsqrt((v * v).mean(1) + EPS)
        y = v * rstd[:, None] * s["weight"].float()
        if s["bias"] is not None:
            y = y + s["bias"].float()
        return dict(y=y.to(dt), mean=mean, rstd=rstd)
    if path == "norm_grad":
        v = _values(s["q"], s["e"], c["dim"]) if c["kept"] else s["x"].float()
        if s["mean"] is not None:
            v = v - s["mean"][:, None]
        v = v * s["rstd"][:, None]
        dy = s["dy"].float()
        a = dy * s["weight"].float()
        dx = a - v * (a * v).mean(1, keepdim=True)
        if s["mean"] is not None:
            dx = dx - a.mean(1, keepdim=True)
        return dict(dx=(dx * s["rstd"][:, None]).to(dt), dweight=(dy * v).sum(0),
                    dbias=dy.sum(0) if s["bias"] is not None else None)
    if path == "save":
        q, e = _quantize(s["x"])
        return dict(x=_values(q, e, c["dim"]).to(dt))
    return dict(dw=torch.matmul(s["dy"].float().t(), _values(s["q"], s["e"], c["dim"])).to(_DT[c["grad"]]))


# --- the same in 64 bits, from the definitions ----------------------------------------------------------------

def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    path, t, d = c["path"], c["tokens"], c["dim"]
    if path == "embed":
        return dict(y=torch.nn.functional.embedding(s["ids"], s["table"].double()) * c["scale"])
    if path == "embed_grad":
        # sums over a row's tokens as differences of one running sum would cancel: a product with the incidence
        # matrix of the rows that have tokens instead, some thousand tokens at a time
        grad = torch.zeros(c["vocab"], d, dtype=torch.float64, device="cuda")
        keep = s["ids"] >= 0
        words, at = torch.unique(s["ids"][keep], return_inverse=True)
        dy = s["dy"][keep].double()
        part = torch.zeros(words.numel(), d, dtype=torch.float64, device="cuda")
        for i in range(0, at.numel(), 4096):
            hit = torch.zeros(words.numel(), min(4096, at.numel() - i), dtype=torch.float64, device="cuda")
            hit[at[i:i + 4096], torch.arange(hit.shape[1], device="cuda")] = c["scale"]
            part += hit @ dy[i:i + 4096]
        grad[words] = part
        return dict(grad=grad)
    if path == "norm":
        x = s["x"].double()
        mean = x.sum(1) / d if c["kind"] == "layer" else None
        var = (x * x).sum(1) / d if mean is None else ((x - mean[:, None]) ** 2).sum(1) / d
        rstd = 1 / (var + EPS).sqrt()
        y = (x if mean is None else x - mean[:, None]) * rstd[:, None] * s["weight"].double()
        return dict(y=y if s["bias"] is None else y + s["bias"].double(), mean=mean, rstd=rstd)
    if path == "norm_grad":
        x = _values(s["q"], s["e"], d, torch.float64) if c["kept"] else s["x"].double()
        rstd, dy, w = s["rstd"].double()[:, None], s["dy"].double(), s["weight"].double()
        xhat = (x if s["mean"] is None else x - s["mean"].double()[:, None]) * rstd
        a = dy * w
        dx = a - xhat * ((a * xhat).sum(1, keepdim=True) / d)
        if s["mean"] is not None:
            dx -= a.sum(1, keepdim=True) / d
        return dict(dx=dx * rstd, dweight=(dy * xhat).sum(0), dbias=None if s["bias"] is None else dy.sum(0))
    if path == "save":
        # the definition, block by block on whole columns: the smallest power of two (from 2^-126) with which 127
        # steps reach the block's largest value, and the nearest of those steps, halves to the even one
        x = s["x"].double()
        out = torch.empty_like(x)
        for b in range(0, d, BLOCK):
            v = x[:, b:b + BLOCK]
            step = torch.exp2(torch.ceil(torch.log2(v.abs().amax(1, keepdim=True).clamp_min(2.0 ** -140) / 127)))
            step = torch.where(step * 63.5 >= v.abs().amax(1, keepdim=True), step / 2, step)    # log2's rounding
            step = torch.where(step * 127 < v.abs().amax(1, keepdim=True), step * 2, step).clamp_min(2.0 ** -126)
            out[:, b:b + BLOCK] = torch.round(v / step) * step
        return dict(x=out)
    x, dy = _values(s["q"], s["e"], d, torch.float64), s["dy"].double()
    return dict(dw=torch.einsum("tn,tk->nk", dy, x))


# --- what a pass cannot do without ----------------------------------------------------------------------------

def _distinct(t, vocab):
    """How many different words t word-like ids hold on average: the sum over k of 1 - exp(-t / (k ln vocab))."""
    a, steps = t / math.log(vocab), 400
    total = 0.0
    for i in range(steps):
        lo, hi = vocab ** (i / steps), vocab ** ((i + 1) / steps)
        total += (hi - lo) * -math.expm1(-a / math.sqrt(lo * hi))
    return min(t, total + 1)


def work(case):
    c = dict(case)
    path, t, d = c["path"], c["tokens"], c["dim"]
    e = 2 if c["dtype"] == BF16 else 4
    nb = -(-d // BLOCK)
    act = t * nb * (BLOCK + 1)                      # bytes of a checkpoint
    if path == "embed":
        # a row that several tokens share is read once
        return dict(bytes=8 * t + e * d * (_distinct(t, c["vocab"]) + t), flops=t * d)
    if path == "embed_grad":
        ge = 2 if c["grad"] == BF16 else 4
        return dict(bytes=8 * t + e * d * t * 15 / 16 + ge * d * c["vocab"], flops=2 * t * d)
    if path == "norm":
        layer = c["kind"] == "layer"
        return dict(bytes=2 * e * t * d + 4 * t * (2 if layer else 1) + e * d * (2 if layer else 1), flops=8 * t * d)
    if path == "norm_grad":
        layer = c["kind"] == "layer"
        return dict(bytes=2 * e * t * d + (act if c["kept"] else e * t * d) + 4 * t * (2 if layer else 1) + e * d
                    + 4 * d * (2 if layer else 1), flops=12 * t * d)
    if path == "save":
        return dict(bytes=2 * e * t * d + 2 * act, flops=4 * t * d)
    ge = 2 if c["grad"] == BF16 else 4
    return dict(bytes=act + e * t * c["rows"] + ge * c["rows"] * d, flops=2 * t * c["rows"] * d)
