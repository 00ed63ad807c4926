"""Group scales, the choice of experts and the layer of experts for a few tokens without a GPU: what the C calls refuse, the sizes of
workspaces, and the 64-bit definitions that the GPU tests compare with.  Only calls that return before the first launch are made here."""
import ctypes
import os

import numpy as np
import pytest
import torch

from tests import grouped_reference as ref

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06786_amd", "libmq.so")
OK, NULL, SHAPE, BITS, ALIGN, WORKSPACE = range(6)
P, ODD = 4096, 4104   # pointers nobody follows; the second one is not a multiple of 16
SILU, RESIDUAL, RENORMALIZE, OP_FFN = 16, 32, 256, 11


class Layer(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("gate_up", "down", "alpha_gu", "zero_gu", "alpha_dn", "zero_dn")] + [("r", ctypes.c_int)]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        pytest.fail(f"{LIB} is not built (python -c 'import __graft_entry__ as g; g.build()')")
    lib_ = ctypes.CDLL(LIB)
    vp, i64, ci, u32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint32, ctypes.c_size_t
    lib_.mq_gemv_grouped.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, ci, vp, vp]
    lib_.mq_experts_choose.argtypes = [vp, i64, i64, i64, i64, u32, vp, vp, vp]
    lib_.mq_experts_choose_bwd.argtypes = [vp, i64, vp, vp, vp, i64, i64, i64, u32, vp, vp]
    lib_.mq_experts_ffn.argtypes = [vp, ctypes.POINTER(Layer), vp, vp, i64, i64, i64, i64, i64, i64, u32, vp, vp, sz, vp]
    lib_.mq_workspace_bytes.argtypes = [ci, i64, i64, i64, ci]
    lib_.mq_workspace_bytes.restype = sz
    return lib_


def test_gemv(lib):
    def f(x=P, packed=P, alpha=P, zero=P, B=4, N=32, K=256, group=64, r=4, y=P):
        return lib.mq_gemv_grouped(x, packed, alpha, zero, B, N, K, group, r, y, None)
    assert f(B=0) == f(B=17) == f(B=-1) == f(N=-1) == f(K=0) == f(K=-64) == f(group=0) == f(group=-64) == SHAPE
    assert f(group=512) == f(group=96) == f(K=300) == f(K=(1 << 20) + 64) == f(N=(1 << 25) + 1) == SHAPE
    assert f(r=0) == f(r=1) == f(r=3) == f(r=6) == f(r=9) == BITS
    assert f(group=16) == f(K=240, group=48) == f(group=32, r=2) == f(group=16, r=8) == f(K=192, group=96, r=2) == ALIGN
    assert f(x=None) == f(packed=None) == f(alpha=None) == f(zero=None) == f(y=None) == NULL
    assert f(x=ODD) == f(packed=ODD) == f(alpha=ODD) == f(zero=ODD) == f(y=ODD) == ALIGN
    assert f(N=0) == f(None, None, None, None, N=0, y=None) == OK


def test_choose(lib):
    def f(scores=P, M=4, E=8, ld=8, top=2, flags=0, ids=P, weight=P):
        return lib.mq_experts_choose(scores, M, E, ld, top, flags, ids, weight, None)

    def b(scores=P, M=4, E=8, ld=8, top=2, flags=0, ids=P, weight=P, dweight=P, dscores=P):
        return lib.mq_experts_choose_bwd(scores, ld, ids, weight, dweight, M, E, top, flags, dscores, None)
    for g in (f, b):
        assert g(M=-1) == g(E=0) == g(E=1025, ld=1025) == g(ld=7) == g(top=0) == g(top=9) == g(E=64, ld=64, top=33) == SHAPE
        assert g(M=(1 << 25) + 1) == g(M=1 << 20, ld=1 << 60) == SHAPE
        assert g(flags=1) == g(flags=16) == g(flags=RENORMALIZE | 1) == BITS
        assert g(scores=None) == g(ids=None) == g(weight=None) == NULL
        assert g(scores=4097) == g(ids=ODD) == g(weight=ODD) == ALIGN   # scores: 4 bytes are enough
        assert g(M=0) == g(None, M=0, ids=None, weight=None) == OK
    assert b(dweight=None) == b(dscores=None) == NULL
    assert b(dweight=ODD) == b(dscores=ODD) == ALIGN


def test_layer(lib):
    def f(x=P, B=4, top=2, E=8, d=256, F=128, group=64, flags=0, ids=P, weight=P, y=P, ws=P, ws_bytes=1 << 40, layer=True, r=4, **arrays):
        names = ("gate_up", "down", "alpha_gu", "zero_gu", "alpha_dn", "zero_dn")
        L = Layer(*(arrays.get(n, P) for n in names), r)
        return lib.mq_experts_ffn(x, ctypes.byref(L) if layer else None, ids, weight, B, top, E, d, F, group, flags, y, ws, ws_bytes, None)
    assert f(B=0) == f(B=17) == f(top=0) == f(top=17) == f(E=0) == f(E=1025) == f(d=0) == f(F=0) == f(d=-64) == f(F=-64) == f(group=-1) == SHAPE
    assert f(group=256) == f(group=96) == f(d=(1 << 20) + 64) == f(F=(1 << 20) + 64) == SHAPE
    assert f(group=16) == f(group=32, r=2) == f(group=0, d=240) == f(group=0, F=144) == f(group=0, F=96, r=2) == ALIGN
    assert f(r=3) == f(r=6) == f(r=0) == f(flags=1) == f(flags=128) == f(flags=RENORMALIZE) == f(flags=64 | SILU) == BITS
    assert f(x=None) == f(ids=None) == f(weight=None) == f(y=None) == f(layer=False) == NULL
    assert f(x=ODD) == f(ids=ODD) == f(weight=ODD) == f(y=ODD) == ALIGN
    for name in ("gate_up", "down", "alpha_gu", "zero_gu", "alpha_dn", "zero_dn"):
        assert f(**{name: None}) == NULL and f(**{name: ODD}) == ALIGN
    need = lib.mq_workspace_bytes(OP_FFN, 8, 128, 256, 1)
    assert need >= 8 * 128 * 4
    assert f(ws=None) == f(ws=ODD) == f(ws_bytes=need - 1) == f(ws_bytes=0) == WORKSPACE
    w = lib.mq_workspace_bytes
    assert w(OP_FFN, 0, 128, 256, 1) == w(OP_FFN, 257, 128, 256, 1) == w(OP_FFN, 8, 0, 256, 1) == w(OP_FFN, 8, (1 << 20) + 1, 256, 1) == 0
    assert w(OP_FFN, 256, 1 << 20, 256, 1) >= 256 << 22


def test_reference_packs_as_the_oracle_does(oracle):
    rng = np.random.default_rng(1)
    for r in (8, 4, 2):
        codes = rng.integers(0, 1 << r, (5, 64))
        assert np.array_equal(ref.pack(codes, r), oracle.pack(codes.astype(np.uint8), r))
        assert np.array_equal(ref.unpack(ref.pack(codes, r), 64, r), codes)


def test_reference_choice_against_autograd():
    """The 64-bit definition of the choice and its gradient, against torch's softmax and autograd in 64 bits."""
    rng = np.random.default_rng(2)
    s = rng.standard_normal((20, 9)).astype(np.float32)
    s[3] = -np.inf
    s[5, :7] = -np.inf
    for renormalize in (False, True):
        ids, w, _ = ref.choose(s, 4, renormalize)
        t = torch.from_numpy(s).double().requires_grad_()
        dw = torch.from_numpy(rng.standard_normal((20, 4)))
        want = np.zeros((20, 9))
        for m in range(20):
            live = ids[m] >= 0
            if not live.any():
                assert not w[m].any()
                continue
            at = torch.from_numpy(ids[m][live])
            p = torch.softmax(t[m][at], 0) if renormalize else torch.softmax(t[m], 0)[at]
            assert np.allclose(p.detach().numpy(), w[m][live], atol=1e-14) and (np.diff(p.detach().numpy()) <= 0).all()
            want[m] = torch.autograd.grad((p * dw[m][torch.from_numpy(live)]).sum(), t)[0][m].numpy()
        got, _ = ref.choose_bwd(s, ids, w, dw.numpy(), renormalize)
        assert np.allclose(got, want, atol=1e-14)


def test_reference_product_against_a_dense_one():
    rng = np.random.default_rng(3)
    codes, alpha, zero = rng.integers(0, 16, (7, 96)), rng.random((7, 3)), 100 * rng.random((7, 3))
    x = rng.standard_normal((2, 96))
    w = np.array([[alpha[n, k // 32] * (16 * codes[n, k] - zero[n, k // 32]) for k in range(96)] for n in range(7)])
    y, bar = ref.product(x, codes, alpha, zero, 4)
    assert np.allclose(y, x @ w.T, atol=1e-9) and (bar > 0).all() and bar.max() < 0.02 * np.abs(y).max()
