"""What stands right before and right behind the outputs and the workspace of the layer in 8-bit integers, in every form: nothing of it is
written.  Each buffer lies in the middle of a larger one, at a multiple of 16 bytes that is no multiple of 256, with exactly the bytes that the call
asks for; the rest of the larger one holds a pattern and has to hold it afterwards."""
import numpy as np
import pytest
import torch

from tests import int8_plans
from tests.test_gpu_int8_forms import DENSE, EXPERTS, SINGLE, inputs, mq, same_bits  # noqa: F401 (mq is a fixture)

pytestmark = pytest.mark.gpu
BEFORE, AFTER, PATTERN = 4096 + 16, 1 << 16, 0xA5


class Watched:
    """Buffers inside larger ones."""

    def __init__(self):
        self.all = []

    def empty(self, *shape, dtype=torch.bfloat16):
        n = int(np.prod(shape)) * dtype.itemsize
        whole = torch.full((BEFORE + n + AFTER,), PATTERN, dtype=torch.uint8, device="cuda")
        self.all.append((whole, n))
        t = whole[BEFORE:BEFORE + n].view(dtype).view(*shape)
        assert n == 0 or t.data_ptr() % 256 == 16   # (an empty tensor has no pointer)
        return t

    def check(self, what):
        for i, (whole, n) in enumerate(self.all):
            for name, edge in (("before", whole[:BEFORE]), ("behind", whole[BEFORE + n:])):
                bad = (edge != PATTERN).nonzero()
                assert not len(bad), (what, "buffer", i, name, "byte", int(bad[0]))


@pytest.mark.parametrize("case", DENSE)
def test_dense(mq, case):  # noqa: F811
    print(case, flush=True)
    _, _, _, T, N, K, r, gate = case
    x, codes, alpha, zero = inputs(T, 1, N, K, r)
    w = (codes[0], alpha[0], zero[0])
    need = mq.mq_workspace_bytes(mq.MQ_OP_LINEAR_FWD_INT8, T, N, K, 1)
    least = mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_FWD_INT8, T, N, K, 1)
    assert (need > least) == (int8_plans.form(T, N, K).part > 0)
    want = mq.mq_linear_fwd_int8(x, *w, r, gate=gate)
    for nbytes in {need, least}:
        b = Watched()
        y = b.empty(*want.shape)
        mq.mq_linear_fwd_int8(x, *w, r, gate=gate, Y=y, ws=b.empty(nbytes, dtype=torch.uint8))
        assert same_bits(y, want)
        b.check((case, nbytes))
    b = Watched()
    tokens = mq.mq_quantize_tokens(x, b.empty(T, K, dtype=torch.int8), b.empty(T, dtype=torch.float32), b.empty(T, dtype=torch.int32))
    y = b.empty(*want.shape)
    mq.mq_linear_fwd_int8_quantized(*tokens, *w, r, gate=gate, Y=y, ws=b.empty(need, dtype=torch.uint8))
    assert same_bits(y, want)
    b.check(case)


@pytest.mark.parametrize("T,N,K,wide", SINGLE)
@pytest.mark.parametrize("r,gate", [(8, None), (4, "silu")])
def test_single(mq, T, N, K, wide, r, gate):  # noqa: F811
    print(T, N, K, r, gate, flush=True)
    N += N % 2 if gate else 0
    x, codes, alpha, zero = inputs(T, 1, N, K, r)
    w = (codes[0], alpha[0], zero[0])
    b = Watched()
    y = b.empty(T, N // 2 if gate else N)
    mq.mq_linear_fwd_int8(x, *w, r, gate=gate, Y=y, ws=b.empty(mq.mq_workspace_bytes(mq.MQ_OP_LINEAR_FWD_INT8, T, N, K, 1), dtype=torch.uint8))
    assert same_bits(y, mq.mq_linear_fwd_int8_quantized(*mq.mq_quantize_tokens(x), *w, r, gate=gate))
    b.check((T, N, K, r, gate))


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("case", EXPERTS + [("single", 8, [1, 0, 2, 1], 3, 515, 528, 8, None), ("single", 3, [0, 3, 5], 4, 1026, 2064, 8, "gelu")])
def test_experts(mq, case, gather):  # noqa: F811
    """Spare places behind the last expert's stay as they are too."""
    print(case[:2], case[3:], flush=True)
    _, E, counts, M, N, K, r, gate = case
    counts = counts + [0] * (E - len(counts))
    used, spare = sum(counts), 0 if case[0] == "single" else 5
    T = used + spare
    if not gather:
        M = T
    x, codes, alpha, zero = inputs(M, E, N, K, r)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32).cuda()
    rows = torch.arange(T, dtype=torch.int32, device="cuda") * 7 % M if gather else None
    if spare and gather:
        rows[used:] = -1
    b = Watched()
    y = b.empty(T, N // 2 if gate else N)
    y.fill_(3.0)
    ws = b.empty(mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_FWD_INT8, max(M, T), N, K, 1), dtype=torch.uint8)
    mq.mq_experts_fwd_int8(x, offsets, codes, alpha, zero, r, rows=rows, gate=gate, Y=y, ws=ws)
    b.check(case)
    assert bool((y[used:] == 3.0).all())
    first = 0
    for e, n in enumerate(counts):
        if n:
            part = x[rows[first:first + n].long()] if gather else x[first:first + n].clone()
            assert same_bits(y[first:first + n], mq.mq_linear_fwd_int8(part, codes[e], alpha[e].clone(), zero[e].clone(), r, gate=gate)), (case, e)
        first += n


@pytest.mark.parametrize("M,K,pad", [(1, 16, 0), (65, 1024, 8), (3, 1040, 0), (513, 2048, 0), (257, 4112, 0), (5, 16384, 0), (2, 16400, 0), (1, 131072, 0)])
def test_quantize(mq, M, K, pad):  # noqa: F811
    x = inputs(M, 1, 8, K + pad, 8)[0][:, :K]
    b = Watched()
    got = mq.mq_quantize_tokens(x, b.empty(M, K, dtype=torch.int8), b.empty(M, dtype=torch.float32), b.empty(M, dtype=torch.int32))
    b.check((M, K, pad))
    assert all(torch.equal(a, c) for a, c in zip(got, mq.mq_quantize_tokens(x)))


@pytest.mark.parametrize("E", [1, 7, 64, 1024])
@pytest.mark.parametrize("M,top", [(0, 2), (1, 1), (31, 3), (1024, 4), (4097, 1), (5000, 3), (9, 1024)])
def test_route_and_combine(mq, M, top, E):  # noqa: F811
    ids = torch.randint(-1, E + 1, (M, top), generator=torch.Generator().manual_seed(M + E), dtype=torch.int32).cuda()
    b = Watched()
    new = lambda *s, dtype=torch.int32: b.empty(*s, dtype=dtype)   # noqa: E731
    offsets, rows, place = mq.mq_experts_route(ids, E, new(E + 1), new(M * top), new(M, top),
                                               ws=new(mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_ROUTE, M * top, E, 0, 1), dtype=torch.uint8))
    b.check((M, top, E))
    for a, c in zip((offsets, rows, place), mq.mq_experts_route(ids, E)):
        assert torch.equal(a, c)
    if not M or M * top > 16000:
        return
    for N in (8, 13):
        y = torch.randn(M * top, N, generator=torch.Generator().manual_seed(N)).to(torch.bfloat16).cuda()
        weight = torch.rand(M, top, device="cuda")
        out = b.empty(M, N)
        mq.mq_experts_combine(y, place, weight, out=out)
        b.check((M, top, E, N))
        assert same_bits(out, mq.mq_experts_combine(y, place, weight))
