"""The example's training loop: it learns, and a restored run repeats the lost steps bit for bit."""
import importlib.util
import os

import pytest

from tests.conftest import ROOT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def load():
    spec = importlib.util.spec_from_file_location("resume_example", os.path.join(ROOT, "examples", "resume.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_resume_repeats_the_lost_steps():
    losses, again, same = load().main(steps=20, fail_at=17)
    assert losses[-1] < losses[0] and len(again) == 3
    assert again == losses[-3:] and same


def test_gradients_are_those_of_the_loss():
    """Against torch's own backward of the same model in 64 bits.  Both kept activations are off by at most half a
    step of their block (a 127th of the block's largest value, up to twice that), and x, h, dlogits and dx are rounded
    to bf16: relative to the whole gradient 2^-7 and a few 2^-9."""
    ex = load()
    model = ex.Model(vocab=500, dim=128, seed=3)
    ids, targets = ex.batch(1, 500, 96)
    loss = model.gradients(ids, targets)
    E = model.copy[0].double().requires_grad_()
    g = model.copy[1].double().requires_grad_()
    x = torch.where((ids >= 0)[:, None], E[ids.clamp(min=0)] * 128 ** 0.5, 0.0)
    h = x / (x * x).mean(1, keepdim=True).add(1e-5).sqrt() * g
    real = targets >= 0
    want = torch.nn.functional.cross_entropy((h @ E.t())[real], targets[real])
    want.backward()
    assert abs(float(loss) - float(want.detach())) < 2 ** -7 * float(want.detach())
    for got, ref in ((model.grad[0], E.grad), (model.grad[1], g.grad)):
        assert float((got.double() - ref).norm()) < 2 ** -6 * float(ref.norm())
