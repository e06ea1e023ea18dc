"""Operators of a training step around the fused optimizer: the embedding
lookup, layer and root-mean-square norms, activations kept in 8 bits for the
backward pass, and the gradients of them that adamw_step_measure reads.

Thin binding of the lc_embed / lc_norm / lc_act / lc_weight_grad calls of
include/layercheck.h over torch CUDA tensors; what is done for every call is in
C++ (binding/ops_binding.cpp).  Work is enqueued on torch's current stream,
outputs that are not passed in come from torch's allocator on that stream, and
scratch up to 32 MB is one tensor a device and stream that grows to the largest
call (more is allocated for the call).  A call inside torch.cuda.graph has
scratch of its own from the graph's pool, so graphs may be replayed beside other
calls and one another.  There is no CPU fallback.

Autograd records none of this: the gradients are calls too, for training loops
that write their backward pass themselves and for torch.autograd.Function.
embed and norm refuse inputs that require a gradient while grad mode is on.

Tensors are rows of their last dimension: [tokens, dim] with any row stride
(an expanded row, stride 0, may be an input) and bfloat16 or float32 elements.
"""
import torch

from . import _abi
from ._abi import LC_ACT_BLOCK, LC_BF16, LC_F32, LC_NORM_LAYER, LC_NORM_RMS

_abi.load()               # says how to build what is missing
try:
    from . import _ops
except ImportError as e:
    raise ImportError("the operators' binding is not built for this torch (run __graft_entry__.build() or "
                      "python paper_2609_27193_gb300/build.py)") from e

_ops.set_errors(_abi.LCError, torch.OutOfMemoryError)

__all__ = ["Act", "embed", "embed_grad", "norm", "norm_grad", "act_save", "act_load", "weight_grad"]

_CODE = {torch.bfloat16: LC_BF16, torch.float32: LC_F32}
_KIND = {"layer": LC_NORM_LAYER, "rms": LC_NORM_RMS}


def _dtype(dtype):
    """The code of an output's type, -1 for none given."""
    if dtype is None:
        return -1
    code = _CODE.get(dtype)
    if code is None:
        raise TypeError("outputs are bfloat16 or float32, not %s" % dtype)
    return code


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
    def _of(cls, q, e, dim):
        act = cls.__new__(cls)
        act.q, act.e, act.dim = q, e, dim
        return act

    @classmethod
    def empty(cls, rows, dim, device):
        blocks = -(-int(dim) // LC_ACT_BLOCK)
        return cls._of(torch.empty((rows, blocks * LC_ACT_BLOCK), dtype=torch.int8, device=device),
                       torch.empty((rows, blocks), dtype=torch.int8, device=device), int(dim))

    @property
    def rows(self):
        return self.q.shape[0]

    @property
    def nbytes(self):
        return self.q.numel() + self.e.numel()


def _for(act, x):
    """The checkpoint that x goes into: the one given, if it is as large, or a new one."""
    if act is None or act is True:
        q, e = _ops.new_act(x)
        return Act._of(q, e, x.shape[1])
    if x.dim() != 2 or (act.rows, act.dim) != x.shape:
        raise ValueError("the checkpoint must have x's %s rows and columns" % (tuple(x.shape),))
    return act


def embed(table, ids, scale=1.0, out=None):
    """scale * table[ids]: [tokens, dim] in the table's type.  A negative id
    gives a zero row, an id beyond the table a row of NaN."""
    return _ops.embed(table, ids, scale, out)


def embed_grad(dy, ids, vocab=None, scale=1.0, grad=None, dtype=None, skip_id=-1, accumulate=False):
    """The gradient of embed's table, [vocab, dim]: row v is scale times the sum
    of dy over the tokens with id v, in a fixed order; the other rows are zero.
    With accumulate the sums are added to `grad` and the other rows stay."""
    return _ops.embed_grad(dy, ids, -1 if vocab is None else vocab, scale, grad, _dtype(dtype), skip_id, accumulate)


def act_save(x, act=None):
    """Keeps x in 8 bits (see Act); `act` is written if given."""
    act = _for(act, x)
    _ops.act_save(x, act.q, act.e)
    return act


def act_load(act, out=None, dtype=torch.bfloat16):
    """The values of a checkpoint, exact in bfloat16 and in float32."""
    return _ops.act_load(act.q, act.e, act.dim, out, _dtype(dtype))


def norm(x, weight, bias=None, eps=1e-5, kind="layer", out=None, keep=None):
    """Layer norm ("layer") or root-mean-square norm ("rms") of every row of x.
    Returns (y, mean, rstd), the statistics fp32 (mean None for "rms").  keep:
    an Act that receives x in 8 bits on the same pass, or True for a new one,
    returned as a fourth value."""
    if keep is None:
        return _ops.norm(x, weight, bias, eps, _KIND[kind], out, None, None)
    act = _for(keep, x)
    result = _ops.norm(x, weight, bias, eps, _KIND[kind], out, act.q, act.e)
    return (*result, act) if keep is True else result


def norm_grad(dy, x, weight, mean, rstd, bias=False, dx=None, dweight=None, dbias=None, dtype=torch.float32,
              accumulate=False):
    """Gradients of norm: (dx, dweight, dbias), dbias None unless `bias` or a
    buffer for it is given.  x: the norm's input, or its checkpoint (Act).
    mean None: the root-mean-square norm.  dweight and dbias are of `dtype`
    where they are made here; accumulate adds to the ones given."""
    if isinstance(x, Act):
        return _ops.norm_grad(dy, None, x.q, x.e, x.dim, weight, mean, rstd, bias, dx, dweight, dbias, _dtype(dtype),
                              accumulate)
    return _ops.norm_grad(dy, x, None, None, 0, weight, mean, rstd, bias, dx, dweight, dbias, _dtype(dtype), accumulate)


def weight_grad(dy, act, grad=None, dtype=torch.float32, accumulate=False):
    """dy^T x for a linear layer's weight [rows of dy, act.dim], with the
    layer's input read from its checkpoint; accumulate adds to `grad`."""
    return _ops.weight_grad(dy, act.q, act.e, act.dim, grad, _dtype(dtype), accumulate)
