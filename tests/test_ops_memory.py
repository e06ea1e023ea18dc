"""Every operator looks at what is behind a tensor before it passes the address on: a storage that was released, or cut
below what the tensor reaches, is refused.  On host tensors, where what comes after that check is "the operators need CUDA
tensors"."""
import pytest

torch = pytest.importorskip("torch")

BF, F32 = torch.bfloat16, torch.float32
T, D = 4, 256


@pytest.fixture(scope="module")
def ops():
    from paper_2609_27193_gb300 import build as B
    B.build()
    from paper_2609_27193_gb300 import ops
    return ops


def tensors():
    return dict(x=torch.zeros(T, D, dtype=BF), r=torch.zeros(T, D), w=torch.ones(D), b=torch.ones(D), mean=torch.zeros(T), rstd=torch.ones(T),
                y=torch.zeros(T, D, dtype=BF), s=torch.zeros(T, D), table=torch.zeros(9, D), ids=torch.zeros(T, dtype=torch.int64), grad=torch.zeros(9, D),
                dw=torch.zeros(D), db=torch.zeros(D), q=torch.zeros(T, D, dtype=torch.int8), e=torch.zeros(T, D // 128, dtype=torch.int8),
                q2=torch.zeros(T, D, dtype=torch.int8), e2=torch.zeros(T, D // 128, dtype=torch.int8), wg=torch.zeros(D, D),
                u=torch.zeros(2, 30, 40), m=torch.zeros(2, 30, 40), o=torch.zeros(2, 30, 40, dtype=BF))


def calls(ops):
    """Every operator, and the tensors that it takes."""
    def act(t, k=""):
        return ops.Act(t["q" + k], t["e" + k], D)
    return {
        "embed": (lambda t: ops.embed(t["table"], t["ids"], out=t["r"]), "table ids r"),
        "embed_grad": (lambda t: ops.embed_grad(t["r"], t["ids"], grad=t["grad"]), "r ids grad"),
        "norm": (lambda t: ops.norm(t["x"], t["w"], t["b"], out=t["y"], keep=act(t)), "x w b y q e"),
        "norm_grad": (lambda t: ops.norm_grad(t["y"], t["x"], t["w"], t["mean"], t["rstd"], dx=t["s"], dweight=t["dw"], dbias=t["db"]),
                      "y x w mean rstd s dw db"),
        "norm_grad of a checkpoint": (lambda t: ops.norm_grad(t["y"], act(t), t["w"], t["mean"], t["rstd"]), "y q e w mean rstd"),
        "act_save": (lambda t: ops.act_save(t["x"], act(t)), "x q e"),
        "act_load": (lambda t: ops.act_load(act(t), out=t["y"]), "q e y"),
        "add_norm": (lambda t: ops.add_norm(t["x"], t["r"], t["w"], out=t["y"], sum=t["s"], keep=act(t), out8=act(t, "2")),
                     "x r w y s q e q2 e2"),
        "add_norm_grad": (lambda t: ops.add_norm_grad(t["y"], t["r"], t["s"], t["w"], t["rstd"], dx=t["grad"][:T], dweight=t["dw"]),
                          "y r s w rstd dw"),
        "add_norm_grad of a checkpoint": (lambda t: ops.add_norm_grad(t["y"], t["r"], act(t), t["w"], t["rstd"]), "y r q e w rstd"),
        "weight_grad": (lambda t: ops.weight_grad(t["x"], act(t), grad=t["wg"]), "x q e wg"),
        "orthogonalize": (lambda t: ops.orthogonalize(t["u"], momentum=t["m"], out=t["o"]), "u m o"),
    }


def views(t):
    """The same shape at the start of its storage, and from some elements on with rows further apart."""
    yield t
    wide = torch.zeros(7 + (t.numel() // t.shape[-1]) * (t.shape[-1] + 3), dtype=t.dtype)
    yield wide[7:].view(*t.shape[:-1], t.shape[-1] + 3)[..., :t.shape[-1]] if t.dim() > 1 else wide[7:7 + t.numel()]


def reach(t):
    """Bytes of a storage up to a tensor's last element."""
    return (t.storage_offset() + 1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride()))) * t.element_size()


NAMES = ["embed", "embed_grad", "norm", "norm_grad", "norm_grad of a checkpoint", "act_save", "act_load", "add_norm", "add_norm_grad",
         "add_norm_grad of a checkpoint", "weight_grad", "orthogonalize"]


@pytest.mark.parametrize("name", NAMES)
def test_every_tensor_of_a_call(ops, name):
    from paper_2609_27193_gb300._abi import LC_ERR_INVALID_ARG, LCError
    call, takes = calls(ops)[name]
    for arg in takes.split():
        for at in range(2):
            t = tensors()
            t[arg] = list(views(t[arg]))[at]
            with pytest.raises(ValueError, match="CUDA tensors"):
                call(t)
            store, last = t[arg].untyped_storage(), reach(t[arg])
            assert store.nbytes() >= last
            # to the byte, one byte less, nothing
            for size in (last, last - 1, 0):
                store.resize_(size)
                with pytest.raises(ValueError if size == last else LCError, match="CUDA tensors" if size == last else "storage") as at_fault:
                    call(t)
                if size < last:
                    assert at_fault.value.status == LC_ERR_INVALID_ARG


def test_tensors_without_elements_reach_nothing(ops):
    x = torch.zeros(3, D)
    x.untyped_storage().resize_(0)
    w = torch.ones(D)
    with pytest.raises(ValueError, match="CUDA tensors"):
        ops.norm(x[:0], w)
    # one row for all of them reaches one row
    row = torch.zeros(1, D).expand(1 << 40, D)
    with pytest.raises(ValueError, match="CUDA tensors"):
        ops.norm(row, w)


def test_meta_tensors(ops):
    with pytest.raises(ValueError, match="CUDA tensors"):
        ops.norm(torch.zeros(3, D, device="meta"), torch.ones(D))
