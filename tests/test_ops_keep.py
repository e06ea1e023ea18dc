"""What add_norm takes for keep and out8: nothing, True, or a checkpoint to write.  On host tensors, where a call that is
taken ends with "the operators need CUDA tensors"."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import build as B
    B.build()
    from paper_2609_27193_gb300 import ops
    return ops


class Truthy:
    def __bool__(self):
        return True


@pytest.mark.parametrize("name", ["keep", "out8"])
def test_what_is_no_checkpoint(ops, name):
    """A value that asks for a checkpoint and is none is refused; it used to be passed over without one."""
    x, w = torch.zeros(4, 64), torch.ones(64)
    q, e = torch.zeros(4, 128, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.int8)
    for bad in (1, 2.0, "yes", (q, e), [True], Truthy(), torch.ones(()), q):
        with pytest.raises(TypeError, match=name):
            ops.add_norm(x, x, w, **{name: bad})
        with pytest.raises(TypeError, match=name):
            ops.add_norm(x, x, w, **{"keep": True, "out8": True, name: bad})
    for good in (None, False, 0, True, ops.Act(q, e, 64)):
        with pytest.raises(ValueError, match="CUDA tensors"):
            ops.add_norm(x, x, w, **{name: good})
