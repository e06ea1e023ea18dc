"""Operators of a training step around the fused optimizer: the embedding
lookup, layer and root-mean-square norms, the norm of a residual sum, activations
kept in 8 bits for the backward pass, the gradients of them that
adamw_step_measure reads, and updates of matrices made orthogonal.

Thin binding of the lc_embed / lc_norm / lc_add_norm / lc_act / lc_weight_grad /
lc_orthogonalize calls of include/layercheck.h over torch CUDA tensors; what is done for every call is in
C++ (binding/ops_binding.cpp).  Work is enqueued on torch's current stream,
outputs that are not passed in come from torch's allocator on that stream, and
scratch up to 32 MB is one tensor a device and stream that grows to the largest
call (more is allocated for the call).  A call inside torch.cuda.graph has
scratch of its own from the graph's pool, so graphs may be replayed beside other
calls and one another.  There is no CPU fallback.

Autograd records none of this: the gradients are calls too, for training loops
that write their backward pass themselves and for torch.autograd.Function.
embed, norm, add_norm and orthogonalize refuse inputs that require a gradient while
grad mode is on.  A tensor whose storage was released, or holds less than the tensor
reaches, is refused by every call, and so is memory that is not device memory.

Tensors are rows of their last dimension: [tokens, dim] with any row stride
(an expanded row, stride 0, may be an input) and bfloat16 or float32 elements;
updates of matrices are [rows, cols] or [batch, rows, cols].
"""
import functools
import struct

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

__all__ = ["Act", "embed", "embed_grad", "norm", "norm_grad", "act_save", "act_load", "add_norm", "add_norm_grad",
           "weight_grad", "orthogonalize"]

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


def _given(name, act, x):
    """The checkpoint that was given to be written; None for a new one (True) and for none."""
    if isinstance(act, Act):
        return _for(act, x)
    if act is not True and (isinstance(act, torch.Tensor) or act):
        raise TypeError("%s must be True or an Act, not %s" % (name, type(act).__name__))
    return None


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


def add_norm(x, residual, weight, eps=1e-5, out=None, sum=None, keep=None, out8=None):
    """The residual sum x + residual and its root-mean-square norm y, in one pass.  Returns (sum, y, rstd), and after
    them the checkpoints made here: keep=True keeps the sum in 8 bits, out8=True keeps y; either may be an Act that
    is written.  sum: where the sum goes, the residual itself if wanted.  out=False: y is wanted in 8 bits only (and
    returned as None).  The sum has the residual's type and y has x's: both the same, or a float32 residual around
    bfloat16 branches."""
    if (keep is None or keep is False) and (out8 is None or out8 is False):
        return _ops.add_norm(x, residual, weight, eps, None if out is False else out, out is not False, sum,
                             None, None, None, None, False, False)
    kept, y8 = _given("keep", keep, x), _given("out8", out8, x)
    result = _ops.add_norm(x, residual, weight, eps, None if out is False else out, out is not False, sum,
                           *((None, None) if kept is None else (kept.q, kept.e)),
                           *((None, None) if y8 is None else (y8.q, y8.e)), keep is True, out8 is True)
    if len(result) == 3:
        return result
    made = tuple(Act._of(result[k], result[k + 1], x.shape[1]) for k in range(3, len(result), 2))
    return (*result[:3], *made)


def add_norm_grad(dy, dsum, total, weight, rstd, dx=None, dweight=None, dtype=torch.float32, accumulate=False):
    """Gradients of add_norm: (dx, dweight).  dx belongs to x and to the residual alike: what comes through the norm
    from dy, and dsum, the sum's own gradient; dx may be dsum itself.  total: the sum, or its checkpoint (Act).
    dweight is of `dtype` where it is made here; accumulate adds to the one given."""
    if isinstance(total, Act):
        return _ops.add_norm_grad(dy, dsum, None, total.q, total.e, total.dim, weight, rstd, dx, dweight, _dtype(dtype),
                                  accumulate)
    return _ops.add_norm_grad(dy, dsum, total, None, None, 0, weight, rstd, dx, dweight, _dtype(dtype), accumulate)


def weight_grad(dy, act, grad=None, dtype=torch.float32, accumulate=False):
    """dy^T x for a linear layer's weight [rows of dy, act.dim], with the
    layer's input read from its checkpoint; accumulate adds to `grad`."""
    return _ops.weight_grad(dy, act.q, act.e, act.dim, grad, _dtype(dtype), accumulate)


@functools.lru_cache(maxsize=64)
def _packed(steps, coefficients):
    """The coefficients of every step as the library takes them: three doubles each."""
    if not 1 <= steps <= 16:
        raise ValueError("1 to 16 steps, not %d" % steps)
    every = coefficients if coefficients and isinstance(coefficients[0], tuple) else (coefficients,) * steps
    if len(every) != steps or any(not isinstance(c, tuple) or len(c) != 3 for c in every):
        raise ValueError("three coefficients for every step, or for each of %d" % steps)
    return struct.pack("%dd" % (3 * steps), *(x for c in every for x in c))


def orthogonalize(update, momentum=None, beta=0.95, nesterov=True, steps=5, coefficients=(3.4445, -4.7750, 2.0315),
                  eps=1e-7, out=None):
    """The update of a weight matrix, [rows, cols], or of a batch of them, [batch, rows, cols], made nearly orthogonal:
    X = U / (|U| + eps), then `steps` times A = X X^T, X = a X + (b A + c A^2) X, returned as bfloat16.  The products take
    fp16 operands; X itself, sums, the diagonals of A and of b A + c A^2 and the norm are held in 32 bits, which leaves the result
    off by some 1e-3 of its norm before its rounding (2.4e-3 for a matrix of rank one).  coefficients: (a, b, c), or a
    sequence of one triple a step.  U is the update, or with `momentum` (float32, written) what comes of it:
    momentum += (1 - beta) (update - momentum), and U = update + beta (momentum - update), without nesterov the
    momentum itself.  update, momentum and out may have any row and batch strides, but none may lie between another's
    first and last element."""
    if not isinstance(coefficients, tuple) or not all(isinstance(c, (int, float, tuple)) for c in coefficients):
        coefficients = tuple(tuple(c) if hasattr(c, "__len__") else c for c in coefficients)
    return _ops.orthogonalize(update, momentum, beta, nesterov, _packed(steps, coefficients), eps, out)
