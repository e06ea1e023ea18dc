"""Tensors whose memory is not from torch's allocators: the operators ask the driver what it is.  Device memory is as good
as torch's, managed memory is refused; both as torch sees them through __cuda_array_interface__."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_ops import BF, gen, randn  # noqa: E402

BYTES = 1 << 20


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import ops
    return ops


@pytest.fixture
def memory():
    """take(managed, like): a tensor of like's shape, type and contents in memory of its own."""
    torch.cuda.init()
    rt = None
    for name in ("libcudart.so.13", "libcudart.so", "/usr/local/cuda/lib64/libcudart.so"):
        try:
            rt = C.CDLL(name)
            break
        except OSError:
            continue
    if rt is None:
        pytest.skip("no shared CUDA runtime to allocate with")
    blocks = []

    def take(managed, like):
        p = C.c_void_p()
        assert (rt.cudaMallocManaged(C.byref(p), C.c_size_t(BYTES), C.c_uint(1)) if managed
                else rt.cudaMalloc(C.byref(p), C.c_size_t(BYTES))) == 0
        blocks.append(p)

        class Block:
            __cuda_array_interface__ = dict(shape=(BYTES,), typestr="|u1", data=(p.value, False), version=2)
        n = like.numel() * like.element_size()
        t = torch.as_tensor(Block(), device="cuda")[:n].view(like.dtype).view(like.shape)
        assert t.data_ptr() == p.value and n <= BYTES
        t.copy_(like)
        return t
    yield take
    torch.cuda.synchronize()
    for p in blocks:
        assert rt.cudaFree(p) == 0


def calls(ops, t):
    """A call a place: (name of the tensor, call, its outputs)."""
    return {
        "x": lambda: ops.norm(t["x"], t["w"])[0],
        "w": lambda: ops.norm(t["x"], t["w"])[0],
        "out": lambda: ops.norm(t["x"], t["w"], out=t["out"])[0],
        "ids": lambda: ops.embed(t["x"], t["ids"]),
        "r": lambda: ops.add_norm(t["x"], t["r"], t["w"])[0],
        "rstd": lambda: ops.add_norm_grad(t["x"], t["r"], t["r"], t["w"], t["rstd"])[1],
        "q": lambda: ops.act_load(ops.Act(t["q"], t["e"], 256)),
        "e": lambda: ops.weight_grad(t["x"], ops.Act(t["q"], t["e"], 256)),
        "u": lambda: ops.orthogonalize(t["u"], momentum=t["m"].clone()),
        "m": lambda: (ops.orthogonalize(t["u"], momentum=t["m"]), t["m"])[1],
    }


def tensors(ops):
    g = gen(71)
    t, d = 40, 256
    act = ops.act_save(randn(g, t, d, dtype=BF))
    return dict(x=randn(g, t, d, dtype=BF), r=randn(g, t, d, dtype=BF), w=randn(g, d), out=torch.zeros(t, d, dtype=BF, device="cuda"),
                ids=torch.arange(t, device="cuda"), rstd=torch.ones(t, device="cuda"), q=act.q, e=act.e, u=randn(g, 90, 130), m=randn(g, 90, 130))


@pytest.mark.parametrize("name", ["x", "w", "out", "ids", "r", "rstd", "q", "e", "u", "m"])
def test_memory_of_another_origin(ops, memory, name):
    from paper_2609_27193_gb300._abi import LCError
    own = tensors(ops)
    first = own[name].clone()
    want = calls(ops, own)[name]().clone()
    own = {**own, name: first}
    managed = {**own, name: memory(True, first)}
    with pytest.raises(LCError, match="device memory"):
        calls(ops, managed)[name]()
    device = {**own, name: memory(False, first)}
    assert torch.equal(calls(ops, device)[name](), want)
    with pytest.raises(LCError, match="device memory"):
        calls(ops, managed)[name]()
    assert torch.equal(calls(ops, own)[name](), want)
