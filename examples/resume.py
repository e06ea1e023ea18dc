"""A training loop through the library's operators, its optimizer step and its checkpoints, and a recovery.

The model is the smallest that has every piece: a token embedding, a root-mean-square norm and the embedding again
as output projection (tied weights), trained to predict the next token.  A step is

  x = embed(E, ids, sqrt(d))             lookup; positions without a token are zero
  h = norm(x, g)                         x is kept in 8 bits on the same pass
  loss of h E^T (torch)                  h is kept in 8 bits
  dE  = weight_grad(dlogits, h kept)     the output projection's part
  dx, dg = norm_grad(dh, x kept)
  dE += embed_grad(dx, ids)              the lookup's part, added
  adamw_step_measure, select, pack_async, commit

Gradients are summed in a fixed order, so a run that is restored from a checkpoint repeats the lost steps bit for
bit; main() checks that.  Run it on a GPU: python examples/resume.py
"""
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_27193_gb300 as P  # noqa: E402
from paper_2609_27193_gb300 import ops  # noqa: E402

EMBED, NORM = 0, 1        # the layers


class Model:
    """fp32 weights with their moments and gradients, and the bf16 copies that the operators read."""

    def __init__(self, vocab=8000, dim=256, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.dim, self.device = vocab, dim, device
        self.w = [0.02 * torch.randn(vocab, dim, generator=g, device=device), torch.ones(dim, device=device)]
        self.copy = [w.to(torch.bfloat16) for w in self.w]
        self.m, self.v, self.grad, self.snap = ([torch.zeros_like(w) for w in self.w] for _ in range(4))
        for s, w in zip(self.snap, self.w):
            s.copy_(w)
        self.register()

    def register(self):
        self.lc = P.LayerCheck(mode=P.LC_DRIFT_ACCUMULATE)
        self.lc.register_layout([P.segment(k, w, s, m, v) for k, (w, s, m, v)
                                 in enumerate(zip(self.w, self.snap, self.m, self.v))], 2, tau_mult=[10.0, 1.0])
        self.lc.register_optimizer(self.grad, self.copy)

    def gradients(self, ids, targets):
        """Loss, and the gradients of both layers into self.grad.  ids, targets: [tokens], -1 for none."""
        E, g = self.copy
        scale = math.sqrt(self.dim)
        x = ops.embed(E, ids, scale=scale)
        h, _, rstd, x_kept = ops.norm(x, g, kind="rms", keep=True)
        h_kept = ops.act_save(h)
        del x
        real = targets >= 0
        logits = (h @ E.t()).float()
        logp = torch.log_softmax(logits, 1)
        at = torch.where(real, targets, 0)
        n = real.sum()
        loss = -(logp.gather(1, at[:, None])[:, 0] * real).sum() / n
        d = logp.exp_()
        d.scatter_add_(1, at[:, None], torch.full_like(d[:, :1], -1.0))
        d = (d * (real / n)[:, None]).to(torch.bfloat16)
        ops.weight_grad(d, h_kept, grad=self.grad[EMBED])
        dx, _, _ = ops.norm_grad(d @ E, x_kept, g, None, rstd, dweight=self.grad[NORM])
        ops.embed_grad(dx, ids, scale=scale, grad=self.grad[EMBED], accumulate=True)
        return loss

    def step(self, t, ids, targets, store, tau=1e-3, max_staleness=4):
        loss = self.gradients(ids, targets)
        self.lc.adamw_step_measure(t, lr=1e-2, weight_decay=0.01)
        mask, _, _ = self.lc.select(tau, max_staleness)
        self.lc.pack_async(store)
        self.lc.commit_snapshot()
        self.lc.wait_durable(t)
        return loss, mask

    def restore(self, store, t_fail):
        steps = self.lc.restore(store, t_fail)
        for c, w in zip(self.copy, self.w):
            c.copy_(w)
        return steps


def batch(t, vocab, tokens, device="cuda"):
    """Step t's tokens and what follows each; the last eighth of them is padding."""
    rng = np.random.default_rng(1000 + t)
    words = np.minimum((float(vocab) ** rng.random(tokens + 1) - 1).astype(np.int64), vocab - 1)
    ids, targets = words[:-1].copy(), words[1:].copy()
    ids[-tokens // 8:] = targets[-tokens // 8:] = -1
    return torch.from_numpy(ids).to(device), torch.from_numpy(targets).to(device)


def main(steps=24, fail_at=20, tokens=512, vocab=8000, dim=256):
    """Trains `steps` steps, loses everything after `fail_at`, restores and repeats.  Step fail_at persists every
    layer, so that the composite is the state of one step.  Returns (losses, repeated losses, whether the weights
    are the same bits)."""
    model = Model(vocab, dim)
    store = P.Store(model.lc, capacity_bytes=steps * sum(model.lc.layer_block_bytes(k) for k in range(2)) + (1 << 20))
    losses = []
    for t in range(1, steps + 1):
        loss, _ = model.step(t, *batch(t, vocab, tokens), store, max_staleness=0 if t == fail_at else 4)
        losses.append(float(loss))
    final = [w.clone() for w in model.w]
    for w in model.w + model.m + model.v:
        w.fill_(float("nan"))
    at = model.restore(store, fail_at)
    assert (at == fail_at).all(), at
    # a context of its own for what follows, as a restarted process has one, over the restored tensors
    model.lc.close()
    model.register()
    again = []
    store = P.Store(model.lc, capacity_bytes=store.capacity)
    for t in range(fail_at + 1, steps + 1):
        loss, _ = model.step(t, *batch(t, vocab, tokens), store)
        again.append(float(loss))
    same = all(torch.equal(a, b) for a, b in zip(final, model.w))
    return losses, again, same


if __name__ == "__main__":
    first, repeated, same = main()
    print("losses  ", " ".join("%.5f" % x for x in first))
    print("repeated", " ".join("%.5f" % x for x in repeated))
    print("the same bits" if same and first[-len(repeated):] == repeated else "DIFFERENT")
