"""The layer in 8-bit integers without a GPU: the argument checks of its C calls, the sizes of its workspaces, the definition that the
GPU tests compare with.  Only calls that return before the first launch are made here."""
import ctypes
import os

import numpy as np
import pytest

from tests import int8_reference as ref

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06786_amd", "libmq.so")
OK, NULL, SHAPE, BITS, ALIGN, WORKSPACE = range(6)
P, ODD = 4096, 4104   # pointers nobody follows; the second one is not a multiple of 16
GATED, SILU = 128, 16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        pytest.fail(f"{LIB} is not built (python -c 'import __graft_entry__ as g; g.build()')")
    lib_ = ctypes.CDLL(LIB)
    vp, i64, ci, u32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint32, ctypes.c_size_t
    lib_.mq_quantize_tokens.argtypes = [vp, i64, i64, i64, vp, vp, vp, vp]
    lib_.mq_linear_fwd_int8.argtypes = [vp, vp, vp, vp, i64, i64, i64, ci, u32, vp, vp, sz, vp]
    lib_.mq_linear_fwd_int8_quantized.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, ci, u32, vp, vp, sz, vp]
    lib_.mq_experts_route.argtypes = [vp, i64, i64, i64, vp, vp, vp, vp, sz, vp]
    lib_.mq_experts_fwd_int8.argtypes = [vp, i64, vp, vp, vp, vp, vp, i64, i64, i64, i64, ci, u32, vp, vp, sz, vp]
    lib_.mq_experts_combine.argtypes = [vp, vp, vp, i64, i64, i64, i64, vp, vp]
    lib_.mq_workspace_bytes.argtypes = [ci, i64, i64, i64, ci]
    lib_.mq_workspace_bytes.restype = sz
    return lib_


def test_quantize_tokens(lib):
    def f(X=P, M=4, K=64, ldx=64, Xq=P, scale=P, sums=P):
        return lib.mq_quantize_tokens(X, M, K, ldx, Xq, scale, sums, None)
    assert f(M=-1) == f(K=0) == f(K=-16) == f(ldx=48) == f(K=131088, ldx=131088) == f(M=1 << 31) == SHAPE
    assert f(K=40) == f(ldx=68) == ALIGN
    assert f(X=None) == f(Xq=None) == f(scale=None) == f(sums=None) == NULL
    assert f(X=ODD) == f(Xq=ODD) == f(scale=ODD) == f(sums=ODD) == ALIGN
    assert f(M=0) == f(None, M=0, Xq=None, scale=None, sums=None) == OK


def test_linear(lib):
    def f(X=P, codes=P, alpha=P, zero=P, M=4, N=32, K=64, r=8, flags=0, Y=P, ws=P, ws_bytes=1 << 30):
        return lib.mq_linear_fwd_int8(X, codes, alpha, zero, M, N, K, r, flags, Y, ws, ws_bytes, None)

    def q(Xq=P, scale=P, sums=P, codes=P, alpha=P, zero=P, M=4, N=32, K=64, r=8, flags=0, Y=P, ws=None, ws_bytes=0):
        return lib.mq_linear_fwd_int8_quantized(Xq, scale, sums, codes, alpha, zero, M, N, K, r, flags, Y, ws, ws_bytes, None)
    for g in (f, q):
        assert g(M=-1) == g(N=-1) == g(K=0) == g(K=131088) == g(M=(1 << 31) - 255) == g(N=(1 << 31) - 255) == SHAPE
        assert g(r=0) == g(r=9) == BITS
        assert g(flags=1) == g(flags=8) == g(flags=1 << 20) == BITS            # the slice with 2^r + 1 levels is not served here
        assert g(K=72) == g(N=31, flags=GATED) == ALIGN
        assert g(codes=None) == g(alpha=None) == g(zero=None) == g(Y=None) == NULL
        assert g(codes=ODD) == g(alpha=ODD) == g(zero=ODD) == g(Y=ODD) == ALIGN
        assert g(M=0) == g(N=0) == g(M=0, codes=None, alpha=None, zero=None, Y=None) == OK
    assert f(X=None) == NULL and f(X=ODD) == ALIGN
    assert q(Xq=None) == q(scale=None) == q(sums=None) == NULL
    assert q(Xq=ODD) == q(scale=ODD) == q(sums=ODD) == ALIGN
    assert q(ws=ODD, ws_bytes=1 << 20) == WORKSPACE
    assert f(ws=None) == f(ws_bytes=16) == f(ws=ODD) == WORKSPACE
    need = lib.mq_workspace_bytes(8, 4, 32, 64, 1)   # (at this size K is not cut)
    assert f(ws_bytes=need - 1) == WORKSPACE


def test_experts(lib):
    def f(X=P, M=8, rows=P, offsets=P, codes=P, alpha=P, zero=P, T=16, E=4, N=32, K=64, r=8, flags=0, Y=P, ws=P, ws_bytes=1 << 30):
        return lib.mq_experts_fwd_int8(X, M, rows, offsets, codes, alpha, zero, T, E, N, K, r, flags, Y, ws, ws_bytes, None)
    assert f(M=-1) == f(T=-1) == f(N=-1) == f(K=0) == f(E=0) == f(E=1025) == f(T=(1 << 31) - 255) == f(K=131088) == SHAPE
    assert f(rows=None, T=9) == f(M=0) == SHAPE                                # more places than tokens
    assert f(r=0) == f(r=9) == f(flags=4) == BITS
    assert f(K=8) == f(N=33, flags=GATED | SILU) == ALIGN
    assert f(X=None) == f(offsets=None) == f(codes=None) == f(alpha=None) == f(zero=None) == f(Y=None) == NULL
    assert f(X=ODD) == f(offsets=ODD) == f(codes=ODD) == f(rows=ODD) == f(Y=ODD) == ALIGN
    assert f(ws=None) == f(ws_bytes=8) == WORKSPACE
    assert f(T=0) == f(N=0) == f(T=0, M=0) == OK


def test_route(lib):
    def f(ids=P, M=8, top=2, E=4, offsets=P, rows=P, place=P, ws=None, ws_bytes=0):
        return lib.mq_experts_route(ids, M, top, E, offsets, rows, place, ws, ws_bytes, None)
    assert f(M=-1) == f(top=0) == f(top=1025) == f(E=0) == f(E=1025) == f(M=1 << 31) == f(M=1 << 30, top=2) == SHAPE
    assert f(ids=None) == f(offsets=None) == f(rows=None) == f(place=None) == NULL
    assert f(ids=ODD) == f(offsets=ODD) == f(rows=ODD) == f(place=ODD) == ALIGN
    assert f(M=5000) == f(M=5000, ws=P, ws_bytes=16) == f(M=5000, ws=ODD, ws_bytes=1 << 20) == WORKSPACE


def test_combine(lib):
    def f(Y=P, place=P, weight=P, T=16, M=8, top=2, N=64, out=P):
        return lib.mq_experts_combine(Y, place, weight, T, M, top, N, out, None)
    assert f(M=-1) == f(N=-1) == f(T=-1) == f(top=0) == f(M=1 << 31) == SHAPE
    assert f(Y=None) == f(place=None) == f(weight=None) == f(out=None) == NULL
    assert f(Y=ODD) == f(place=ODD) == f(weight=ODD) == f(out=ODD) == ALIGN
    assert f(M=0) == f(N=0) == OK


def test_workspaces(lib):
    f = lib.mq_workspace_bytes
    for op in (8, 10):
        assert f(op, 100, 64, 4096, 1) >= 100 * 4096 + 800
        assert f(op, 100, 64, 131088, 1) == 0 and f(op, -1, 64, 64, 1) == 0 and f(op, 100, 64, 0, 1) == 0
    assert f(10, 100, 64, 4096, 1) <= f(10, 101, 64, 4096, 1)
    assert f(8, 77, 4096, 14336, 1) > f(10, 77, 4096, 14336, 1)      # partial sums
    assert f(8, 4000, 14336, 4096, 1) == f(10, 4000, 14336, 4096, 1)
    assert f(9, 5000, 64, 0, 1) >= 2 * 65 * 4 and f(9, 5000, 0, 0, 1) == 0 and f(9, 5000, 1025, 0, 1) == 0


# ---- the reference itself, on cases done by hand --------------------------------------------------------------------------
def test_reference_tokens():
    x = np.array([[127.0, -63.5, 0.5, 1.5, 2.5], [0, 0, 0, 0, 0], [1, np.inf, 0, 0, 0], [2.0 ** -133, 0, -2.0 ** -133, 0, 0]], np.float32)
    codes, scale, sums = ref.quantize_tokens(x)
    assert codes.tolist() == [[127, -64, 0, 2, 2], [0] * 5, [0] * 5, [127, 0, -127, 0, 0]]
    assert scale[0] == 1 and scale[1] == 0 and np.isnan(scale[2]) and scale[3] > 0 and sums.tolist() == [67, 0, 0, 0]


def test_reference_layer():
    """The outputs are the plain product of dequantized tokens and weights."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 32)).astype(np.float32)
    cx, s, _ = ref.quantize_tokens(x)
    for r in (1, 3, 8):
        c = rng.integers(0, 1 << r, (6, 32))
        a, z = rng.uniform(0.1, 1, 6).astype(np.float32), rng.uniform(100, 150, 6).astype(np.float32)
        y, bar = ref.layer(cx, s, c, a, z, r)
        W = a[:, None].astype(np.float64) * (c * 2.0 ** (8 - r) - z[:, None])
        plain = (cx * s[:, None].astype(np.float64)) @ W.T
        assert np.allclose(y, plain, rtol=1e-12, atol=1e-10)
        ref.within(y, y, bar)
        wrong = y.copy()
        wrong[2, 3] *= 1.01
        with pytest.raises(AssertionError):
            ref.within(wrong, y, bar)


def test_reference_route_and_combine():
    offsets, rows, place = ref.route(np.array([[2, 0], [0, -1], [9, 2]]), 3)
    assert offsets.tolist() == [0, 2, 2, 4] and rows.tolist() == [0, 1, 0, 2, -1, -1] and place.tolist() == [[2, 0], [1, -1], [-1, 3]]
    y = np.arange(8.0).reshape(4, 2)
    out, _ = ref.combine(y, place[:2], np.array([[1.0, 2.0], [3.0, 4.0]], np.float32))
    assert out.tolist() == [[4.0 + 0.0, 5.0 + 2.0], [6.0, 9.0]]
