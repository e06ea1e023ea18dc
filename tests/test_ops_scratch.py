"""The test switch of the operators' waits and the scratch that they ask for, without a GPU."""


def test_flags():
    from paper_2609_27193_gb300 import build as B
    B.build()
    from paper_2609_27193_gb300 import _abi
    lib = _abi.load()
    assert lib.lc_ops_debug(_abi.LC_DEBUG_OPS_STALL) == 0 and lib.lc_ops_debug(0) == 0
    for flags in (1, 2, 8, -1):
        assert lib.lc_ops_debug(flags) == _abi.LC_ERR_INVALID_ARG and b"debug flags" in lib.lc_last_error()


def test_the_weight_gradient_asks_for_what_it_uses():
    """A bf16 dy on 16-byte boundaries is not copied, and nobody holds room for a copy of it."""
    from paper_2609_27193_gb300 import build as B
    B.build()
    from paper_2609_27193_gb300 import _abi
    lib = _abi.load()
    need = lib.lc_weight_grad_workspace_of
    t, n, k = 8192, 4096, 14336
    dy = lambda ptr=4096, stride=n, dtype=_abi.LC_BF16: _abi.lc_rows(ptr, stride, dtype, 0)  # noqa: E731
    any_bf16, any_f32 = (lib.lc_weight_grad_workspace(t, n, k, d) for d in (_abi.LC_BF16, _abi.LC_F32))
    assert any_bf16 == t * n * 2 and any_f32 == 3 * t * n * 2
    assert need(dy(), t, n, k) == 0
    assert need(dy(4096 + 2), t, n, k) == need(dy(stride=n + 1), t, n, k) == need(dy(stride=0), t, n, k) == any_bf16
    assert need(dy(dtype=_abi.LC_F32), t, n, k) == any_f32
    # split tokens have their parts either way
    parts = need(dy(stride=256), 2048, 256, 256)
    assert parts > 0 and parts % (256 * 256 * 4) == 0
    assert lib.lc_weight_grad_workspace(2048, 256, 256, _abi.LC_BF16) == parts + 2048 * 256 * 2
    assert need(None, t, n, k) == 0 and need(dy(), 0, n, k) == 0 and need(dy(dtype=9), t, n, k) == 0
