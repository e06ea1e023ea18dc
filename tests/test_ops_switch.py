"""The test switch of the operators' waits, without a GPU."""


def test_flags():
    from paper_2609_27193_gb300 import build as B
    B.build()
    from paper_2609_27193_gb300 import _abi
    lib = _abi.load()
    assert lib.lc_ops_debug(_abi.LC_DEBUG_OPS_STALL) == 0 and lib.lc_ops_debug(0) == 0
    for flags in (1, 2, 8, -1):
        assert lib.lc_ops_debug(flags) == _abi.LC_ERR_INVALID_ARG and b"debug flags" in lib.lc_last_error()
