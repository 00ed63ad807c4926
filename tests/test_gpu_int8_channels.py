"""Channels whose weights are all the same, in 8-bit integers.  mq_quantize_int8 gives them scale 1, zero-point -w and codes of zero, so that the
weight comes back exactly; then y = scale_m w sum_m whatever the size of w: three fp32 roundings (w sum_m, the sum of both terms, the
token's scale) and one to bf16, with nothing left of the 128 that the matrix core's signed reading takes off a code of 8 bits."""
import numpy as np
import pytest
import torch

from tests import int8_plans, int8_reference as ref
from tests.test_gpu_int8_forms import DENSE, inputs, mq  # noqa: F401 (mq is a fixture)

pytestmark = pytest.mark.gpu

SAME = [0.5, 0.02, -1e-3, 3e-5, -1e-6, 2e-10, 0.0, 1e-30]
# a dense product of each form at 8 bits and at fewer, and single tokens
SIZES = [(c[0], *c[3:7]) for c in DENSE if c[7] is None] + [("single", 1, 4096, 4096, 8), ("single", 2, 12290, 272, 8), ("single", 3, 1027, 400, 4)]


def channels(N):
    """Where the channels of SAME stand: beside each other at both ends, and on their own."""
    n = len(SAME)
    return torch.cat([torch.arange(n), N // 2 + 3 * torch.arange(n), N - n + torch.arange(n)]), torch.tensor(SAME, dtype=torch.float32).repeat(3)


@pytest.mark.parametrize("form,T,N,K,r", SIZES)
def test_channels_of_one_weight(mq, form, T, N, K, r):  # noqa: F811
    print(form, T, N, K, r, flush=True)
    at, w = channels(N)
    x, codes, alpha, zero = (t if i == 0 else t[0] for i, t in enumerate(inputs(T, 1, N, K, r)))
    codes[at.cuda()] = 0
    alpha[at.cuda()], zero[at.cuda()] = 1.0, -w.cuda()
    y = mq.mq_linear_fwd_int8(x, codes, alpha, zero, r)[:, at.cuda()].cpu().double().numpy()
    _, scale, sums = (t.cpu().double().numpy() for t in mq.mq_quantize_tokens(x))
    want = w.double().numpy() * (sums * scale)[:, None]
    bar = (2.0 ** -8 + 4 * 2.0 ** -24) * np.abs(want) + 2.0 ** -133
    ref.within(y, want, bar, (form, T, N, K, r))


def test_as_quantized_by_the_library(mq):  # noqa: F811
    K = 528
    W = torch.randn(40, K, generator=torch.Generator().manual_seed(1)) * 0.02
    W[:len(SAME)] = torch.tensor(SAME)[:, None]
    Q, alpha, zero = mq.mq_quantize_int8(W.cuda())
    x = inputs(70, 1, 8, K, 8)[0]
    _, scale, sums = (t.cpu().double().numpy() for t in mq.mq_quantize_tokens(x))
    want = W[:len(SAME), 0].double().numpy() * (sums * scale)[:, None]
    for r in (8, 4, 2):
        codes = Q if r == 8 else mq.mq_slice(Q, r)
        for first, n in ((0, 70), (0, 1), (30, 8)):
            y = mq.mq_linear_fwd_int8(x[first:first + n].contiguous(), codes, alpha, zero, r)[:, :len(SAME)].cpu().double().numpy()
            part = want[first:first + n]
            ref.within(y, part, (2.0 ** -8 + 4 * 2.0 ** -24) * np.abs(part) + 2.0 ** -133, (r, first))


def test_every_form_is_here():
    assert {s[0] for s in SIZES if s[4] == 8} == set(int8_plans.FORMS) | {"single"}
