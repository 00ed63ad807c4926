"""What the C calls of the layer in 8-bit integers refuse before their first launch, beside tests/test_int8_abi.py (no GPU: nothing is
enqueued by a call that fails, so none is needed)."""
from tests.test_int8_abi import ALIGN, BITS, GATED, P, SHAPE, SILU, lib  # noqa: F401 (lib is a fixture)


def linear(lib, M=4, N=32, K=64, r=8, flags=0, ws=P, ws_bytes=1 << 62):  # noqa: F811
    return lib.mq_linear_fwd_int8(P, P, P, P, M, N, K, r, flags, P, ws, ws_bytes, None)


def quantized(lib, M=4, N=32, K=64, r=8, flags=0, ws=None, ws_bytes=0):  # noqa: F811
    return lib.mq_linear_fwd_int8_quantized(P, P, P, P, P, P, M, N, K, r, flags, P, ws, ws_bytes, None)


def experts(lib, M=8, rows=P, T=16, E=4, N=32, K=64, r=8, flags=0, ws=P, ws_bytes=1 << 62):  # noqa: F811
    return lib.mq_experts_fwd_int8(P, M, rows, P, P, P, P, T, E, N, K, r, flags, P, ws, ws_bytes, None)


def test_the_kind_of_gate_without_a_gate(lib):  # noqa: F811
    """SiLU says which gate; alone it would be a product without one, whose Y is twice as wide as that of the caller who forgot the other flag."""
    for call in (linear, quantized, experts):
        assert call(lib, flags=SILU) == BITS
        assert call(lib, flags=SILU, N=31) == BITS
        assert call(lib, flags=SILU | GATED, N=31) == ALIGN   # the pair is a gate: refused for the odd number of channels only


def test_more_tiles_than_a_launch_counts(lib):  # noqa: F811
    """2^45 outputs and more: refused like any other size, before the tokens are quantized (that launch would come back as DEVICE here)."""
    most = 0x7FFFFF00
    for call in (linear, quantized):
        assert call(lib, M=most, N=most, K=16) == SHAPE
        assert call(lib, M=1 << 24, N=1 << 24, K=4096) == SHAPE
    assert experts(lib, M=most, T=most, E=1024, N=most, K=16) == SHAPE
    assert experts(lib, M=1, T=1 << 20, E=1024, N=most, K=16) == SHAPE


def test_workspaces_of_sizes_that_the_calls_refuse(lib):  # noqa: F811
    """0, as for other invalid arguments, and not what is left of a product that does not fit 64 bits."""
    f, most = lib.mq_workspace_bytes, 0x7FFFFF00
    for op in (8, 10):
        assert f(op, most, 64, 16, 1) > most * 128 and f(op, 4, most, 16, 1) > 0
        assert f(op, most + 1, 64, 16, 1) == f(op, 4, most + 1, 16, 1) == 0
        assert f(op, 1 << 57, 64, 16, 1) == f(op, 1 << 62, 1 << 62, 131072, 1) == 0
        assert f(op, 4, 64, 72, 1) == 0
    assert f(9, most + 1, 64, 0, 1) == f(9, -1, 64, 0, 1) == 0
    assert f(9, 5000, 64, -1, 1) == f(9, 5000, 64, 0, 1) > 0   # (K is not looked at)
