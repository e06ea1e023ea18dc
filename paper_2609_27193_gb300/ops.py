"""Operators of a training step around the fused optimizer: the embedding
lookup, layer and root-mean-square norms, activations kept in 8 bits for the
backward pass, and the gradients of them that adamw_step_measure reads.

Thin binding of the lc_embed / lc_norm / lc_act / lc_weight_grad calls of
include/layercheck.h over torch CUDA tensors.  Work is enqueued on torch's
current stream, outputs that are not passed in come from torch's allocator on
that stream, and scratch is one tensor a device and stream that grows to the
largest call (make the first call of a size before a stream capture).  There
is no CPU fallback.

Tensors are rows of their last dimension: [tokens, dim] with any row stride
(an expanded row, stride 0, may be an input) and bfloat16 or float32 elements.
"""
import ctypes as C

import torch

from . import _abi
from ._abi import LC_ACT_BLOCK, LC_BF16, LC_F32, LC_I32, LC_I64, LC_NORM_LAYER, LC_NORM_RMS, check, lc_act, lc_rows

__all__ = ["Act", "embed", "embed_grad", "norm", "norm_grad", "act_save", "act_load", "weight_grad"]

_CODE = {torch.bfloat16: LC_BF16, torch.float32: LC_F32}
_IDS = {torch.int32: LC_I32, torch.int64: LC_I64}
_KIND = {"layer": LC_NORM_LAYER, "rms": LC_NORM_RMS}
_scratch = {}
_empty, _empty_like = torch.empty, torch.empty_like
_f32 = torch.float32


class Act:
    """An activation of `rows` x `dim` kept in 8 bits.

    q: int8 [rows, blocks * 128], e: int8 [rows, blocks], blocks = ceil(dim / 128).
    Value c of row t is q[t, c] * 2 ** e[t, c // 128]; e = 127 marks a block
    that held a NaN or an infinity (it reads as NaN)."""

    __slots__ = ("q", "e", "dim")

    def __init__(self, q, e, dim):
        blocks = -(-int(dim) // LC_ACT_BLOCK)
        qs, es, qt, et = q.shape, e.shape, q.stride(), e.stride()
        if (q.dtype != torch.int8 or e.dtype != torch.int8 or len(qs) != 2 or len(es) != 2 or dim <= 0
                or qs[1] < blocks * LC_ACT_BLOCK or es[1] < blocks or qs[0] != es[0]
                or qt[1] != 1 or (et[1] != 1 and es[1] > 1)):
            raise ValueError("a checkpoint of width %d has int8 rows of %d values and %d exponents"
                             % (dim, blocks * LC_ACT_BLOCK, blocks))
        if q.device != e.device:
            raise ValueError("q and e must be on one device")
        self.q, self.e, self.dim = q, e, int(dim)

    @classmethod
    def empty(cls, rows, dim, device):
        blocks = -(-int(dim) // LC_ACT_BLOCK)
        act = cls.__new__(cls)
        act.q = _empty((rows, blocks * LC_ACT_BLOCK), dtype=torch.int8, device=device)
        act.e = _empty((rows, blocks), dtype=torch.int8, device=device)
        act.dim = int(dim)
        return act

    @property
    def rows(self):
        return self.q.shape[0]

    @property
    def nbytes(self):
        return self.q.numel() + self.e.numel()

    def _c(self):
        return lc_act(self.q.data_ptr(), self.q.stride(0), self.e.data_ptr(), self.e.stride(0))


def _rows(t, name):
    code = _CODE.get(t.dtype)
    if code is None:
        raise TypeError("%s must be bfloat16 or float32, got %s" % (name, t.dtype))
    stride = t.stride()
    if len(stride) != 2 or (stride[1] != 1 and t.shape[1] > 1):
        raise ValueError("%s must be 2-D with contiguous rows" % name)
    return lc_rows(t.data_ptr(), stride[0], code, 0)


def _on(first, *tensors):
    """The device index that all of them are on."""
    index = first.get_device()
    if index < 0:
        raise ValueError("the operators need CUDA tensors")
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError("every tensor must be on %s" % first.device)
    return index


def _like(x):
    return _empty_like(x) if x.is_contiguous() else _empty(x.shape, dtype=x.dtype, device=x.device)


# the handle of torch's current stream, without a Stream object around it (1 us a call)
_stream = torch._C._cuda_getCurrentRawStream


def _workspace(index, stream, nbytes):
    if not nbytes:
        return None
    w = _scratch.get((index, stream))
    if w is None or w.numel() < nbytes:
        w = _scratch[(index, stream)] = torch.empty(nbytes, dtype=torch.uint8, device="cuda:%d" % index)
    return w.data_ptr()


def _param(t, dim, name):
    if t.dtype not in _CODE:
        raise TypeError("%s must be bfloat16 or float32, got %s" % (name, t.dtype))
    if t.shape != (dim,) or not t.is_contiguous():
        raise ValueError("%s must be contiguous with %d elements" % (name, dim))
    return t.data_ptr()


def _ids(ids):
    if ids.dtype not in _IDS:
        raise TypeError("ids must be int32 or int64, got %s" % ids.dtype)
    if ids.dim() != 1 or not ids.is_contiguous():
        raise ValueError("ids must be 1-D and contiguous")
    return _IDS[ids.dtype]


def _shaped(t, rows, dim, name):
    if t.shape != (rows, dim):
        raise ValueError("%s must have shape [%d, %d]" % (name, rows, dim))


def embed(table, ids, scale=1.0, out=None):
    """scale * table[ids]: [tokens, dim] in the table's type.  A negative id
    gives a zero row, an id beyond the table a row of NaN."""
    index = _on(table, ids, out)
    rt, it = _rows(table, "table"), _ids(ids)
    n, (vocab, dim) = ids.numel(), table.shape
    if out is None:
        out = _empty((n, dim), dtype=table.dtype, device=table.device)
        ro = lc_rows(out.data_ptr(), dim, rt.dtype, 0)
    else:
        _shaped(out, n, dim, "out")
        ro = _rows(out, "out")
    check(_abi.load().lc_embed(index, _stream(index), rt, vocab, dim, ids.data_ptr(), it, n, scale, ro))
    return out


def embed_grad(dy, ids, vocab=None, scale=1.0, grad=None, dtype=None, skip_id=-1, accumulate=False):
    """The gradient of embed's table, [vocab, dim]: row v is scale times the sum
    of dy over the tokens with id v, in token order; the other rows are zero.
    With accumulate the sums are added to `grad` and the other rows stay."""
    index = _on(dy, ids, grad)
    rd, it = _rows(dy, "dy"), _ids(ids)
    n, dim = dy.shape
    if ids.numel() != n:
        raise ValueError("dy and ids must have the same number of tokens")
    if grad is None:
        if accumulate:
            raise ValueError("accumulate needs grad")
        if vocab is None:
            raise ValueError("vocab or grad is needed")
        grad = _empty((vocab, dim), dtype=dtype or dy.dtype, device=dy.device)
    else:
        vocab = grad.shape[0]
        _shaped(grad, vocab, dim, "grad")
    rg = _rows(grad, "grad")
    lib, stream = _abi.load(), _stream(index)
    need = lib.lc_embed_grad_workspace(n, vocab, dim)
    check(lib.lc_embed_grad(index, stream, rd, ids.data_ptr(), it, n, scale, skip_id, rg, vocab, dim,
                            1 if accumulate else 0, _workspace(index, stream, need), need))
    return grad


def act_save(x, act=None):
    """Keeps x in 8 bits (see Act); `act` is written if given."""
    index = _on(x, None if act is None else act.q)
    rx = _rows(x, "x")
    n, dim = x.shape
    if act is None:
        act = Act.empty(n, dim, x.device)
    elif act.rows != n or act.dim != dim:
        raise ValueError("the checkpoint must have %d rows of %d" % (n, dim))
    check(_abi.load().lc_act_save(index, _stream(index), rx, n, dim, act._c()))
    return act


def act_load(act, out=None, dtype=torch.bfloat16):
    """The values of a checkpoint, exact in bfloat16 and in float32."""
    index = _on(act.q, out)
    n, dim = act.q.shape[0], act.dim
    if out is None:
        out = _empty((n, dim), dtype=dtype, device=act.q.device)
    else:
        _shaped(out, n, dim, "out")
    ro = _rows(out, "out")
    check(_abi.load().lc_act_load(index, _stream(index), act._c(), n, dim, ro))
    return out


def norm(x, weight, bias=None, eps=1e-5, kind="layer", out=None, keep=None):
    """Layer norm ("layer") or root-mean-square norm ("rms") of every row of x.
    Returns (y, mean, rstd), the statistics fp32 (mean None for "rms").  keep:
    an Act that receives x in 8 bits on the same pass, or True for a new one,
    returned as a fourth value."""
    device = x.device
    new = keep is True
    if new:
        keep = Act.empty(x.shape[0], x.shape[1], device)
    index = _on(x, weight, bias, out, None if keep is None else keep.q)
    rx = _rows(x, "x")
    n, dim = x.shape
    w = _param(weight, dim, "weight")
    b = None if bias is None else _param(bias, dim, "bias")
    if bias is not None and bias.dtype != weight.dtype:
        raise ValueError("weight and bias must have one type")
    if keep is not None and (keep.rows != n or keep.dim != dim):
        raise ValueError("the checkpoint must have %d rows of %d" % (n, dim))
    if out is None:
        out = _like(x)
        ro = lc_rows(out.data_ptr(), dim, rx.dtype, 0)
    else:
        _shaped(out, n, dim, "out")
        ro = _rows(out, "out")
    kind = _KIND[kind]
    rstd = _empty(n, dtype=_f32, device=device)
    mean = _empty_like(rstd) if kind == LC_NORM_LAYER else None
    check(_abi.load().lc_norm(index, _stream(index), kind, rx, n, dim, w, b, _CODE[weight.dtype], eps, ro,
                              None if mean is None else mean.data_ptr(), rstd.data_ptr(),
                              None if keep is None else keep._c()))
    return (out, mean, rstd, keep) if new else (out, mean, rstd)


def norm_grad(dy, x, weight, mean, rstd, bias=False, dx=None, dweight=None, dbias=None, dtype=torch.float32,
              accumulate=False):
    """Gradients of norm: (dx, dweight, dbias), dbias None unless `bias` or a
    buffer for it is given.  x: the norm's input, or its checkpoint (Act).
    mean None: the root-mean-square norm.  dweight and dbias are of `dtype`
    where they are made here; accumulate adds to the ones given."""
    device = dy.device
    kept = isinstance(x, Act)
    index = _on(dy, x.q if kept else x, weight, mean, rstd, dx, dweight, dbias)
    rd = _rows(dy, "dy")
    n, dim = dy.shape
    w = _param(weight, dim, "weight")
    if (x.rows, x.dim) != (n, dim) if kept else tuple(x.shape) != (n, dim):
        raise ValueError("x must have dy's shape")
    for t in (mean, rstd):
        if t is not None and (t.dtype != _f32 or t.shape != (n,) or not t.is_contiguous()):
            raise ValueError("mean and rstd must be contiguous float32 with %d elements" % n)
    if accumulate and (dweight is None or (bias and dbias is None)):
        raise ValueError("accumulate needs the gradients to add to")
    if dx is None:
        dx = _like(dy)
        rdx = lc_rows(dx.data_ptr(), dim, rd.dtype, 0)
    else:
        _shaped(dx, n, dim, "dx")
        rdx = _rows(dx, "dx")
    if dweight is None:
        dweight = _empty(dim, dtype=dbias.dtype if dbias is not None else dtype, device=device)
    pw = _param(dweight, dim, "dweight")
    pb = None
    if dbias is not None:
        pb = _param(dbias, dim, "dbias")
        if dbias.dtype != dweight.dtype:
            raise ValueError("dweight and dbias must have one type")
    elif bias:
        dbias = _empty_like(dweight)
        pb = dbias.data_ptr()
    lib, stream = _abi.load(), _stream(index)
    need = lib.lc_norm_grad_workspace(n, dim)
    check(lib.lc_norm_grad(index, stream, LC_NORM_RMS if mean is None else LC_NORM_LAYER, rd,
                           None if kept else _rows(x, "x"), x._c() if kept else None, n, dim, w,
                           _CODE[weight.dtype], None if mean is None else mean.data_ptr(), rstd.data_ptr(), rdx, pw,
                           pb, _CODE[dweight.dtype], 1 if accumulate else 0, _workspace(index, stream, need), need))
    return dx, dweight, dbias


def weight_grad(dy, act, grad=None, dtype=torch.float32, accumulate=False):
    """dy^T x for a linear layer's weight [rows of dy, act.dim], with the
    layer's input read from its checkpoint; accumulate adds to `grad`."""
    index = _on(dy, act.q, grad)
    rd = _rows(dy, "dy")
    n, rows = dy.shape
    if act.rows != n:
        raise ValueError("dy and the checkpoint must have the same number of tokens")
    if grad is None:
        if accumulate:
            raise ValueError("accumulate needs grad")
        grad = _empty((rows, act.dim), dtype=dtype, device=dy.device)
    else:
        _shaped(grad, rows, act.dim, "grad")
    rg = _rows(grad, "grad")
    lib, stream = _abi.load(), _stream(index)
    need = lib.lc_weight_grad_workspace(n, rows, act.dim, rd.dtype)
    check(lib.lc_weight_grad(index, stream, rd, act._c(), n, rows, act.dim, rg, 1 if accumulate else 0,
                             _workspace(index, stream, need), need))
    return grad
