"""Every form that a product in 8-bit integers can take (csrc/mq_int8_plan.h), at sizes that the rule gives to it, against the definition in 64
bits; channels, lengths and tokens that end inside blocks, tiles and stages.  All forms have the same bits, so parts of a call are also
compared with calls that take another form."""
import numpy as np
import pytest
import torch

from tests import int8_plans, int8_reference as ref

# (form, whether K is cut, whether a last round of tiles is done in quarters), tokens, channels, values a token, bits, gate
DENSE = [
    ("few", False, False, 16, 333, 1040, 8, None), ("few", False, False, 9, 1028, 2064, 4, "silu"), ("few", False, False, 5, 4099, 4112, 8, None),
    ("mid32", False, False, 50, 4099, 528, 8, None), ("mid32", False, False, 70, 2304, 1040, 4, "gelu"), ("mid32", False, False, 33, 5001, 16, 8, None),
    ("mid32", True, False, 20, 2051, 4112, 8, None), ("mid32", True, False, 30, 4352, 4112, 2, "silu"), ("mid32", True, False, 13, 70, 8208, 8, None),
    ("mid64", False, False, 401, 4099, 528, 8, None), ("mid64", False, False, 180, 9472, 528, 6, "gelu"),
    ("mid64", True, False, 100, 2050, 4112, 8, "gelu"), ("mid64", True, False, 300, 1027, 4112, 3, None),
    ("mid96", False, False, 600, 2051, 4112, 8, None), ("mid96", False, False, 200, 5002, 4112, 5, "silu"),
    ("mid96", True, False, 180, 4352, 8208, 4, "silu"), ("mid96", True, False, 77, 4099, 8208, 8, None),
    ("deep128", False, False, 511, 4099, 1040, 8, None), ("deep128", False, False, 200, 9472, 1040, 4, "gelu"), ("deep128", False, False, 401, 5001, 1040, 8, None),
    ("deep128", True, False, 770, 1027, 8208, 8, None), ("deep128", True, False, 200, 4352, 8208, 6, "silu"), ("deep128", True, False, 255, 4099, 8208, 2, None),
    ("tile128", False, False, 511, 4099, 16, 8, None), ("tile128", False, False, 1030, 5002, 144, 4, "gelu"), ("tile128", False, False, 180, 14335, 272, 8, None),
    ("tile128", False, False, 4100, 5001, 144, 8, None), ("tile128", False, False, 1030, 14336, 272, 8, "silu"),
    ("tile256", False, False, 1030, 9001, 272, 8, None), ("tile256", False, False, 2050, 4352, 272, 7, "gelu"), ("tile256", False, False, 600, 14336, 16, 8, None),
    ("tile256", False, False, 3000, 9001, 144, 8, None), ("tile256", False, False, 3000, 14336, 48, 4, "silu"),
    ("tile256", False, True, 4100, 9001, 272, 8, None), ("tile256", False, True, 4100, 9472, 272, 2, "gelu"), ("tile256", False, True, 4100, 4099, 144, 8, None), ("tile256", False, True, 3900, 4400, 528, 8, None),
]
# tokens, channels, values, whether a workgroup has 32 channels: quantized by the product's own workgroups
SINGLE = [(1, 7, 16, False), (1, 4096, 4096, False), (2, 333, 8208, False), (3, 1027, 16384, False), (1, 14336, 1040, True), (2, 12290, 272, True), (3, 16385, 400, True)]
# form, experts, places of each (the rest have none), tokens, channels, values, bits, gate
EXPERTS = [
    ("few", 8, [5, 0, 0, 1, 0, 3], 7, 1027, 1040, 8, None), ("few", 40, [0] * 36 + [4, 3, 1, 1], 4, 1026, 528, 4, "gelu"), ("few", 3, [40, 1, 49], 60, 1027, 4112, 8, None),
    ("mid32", 8, [3, 0, 9, 1, 0, 0, 17], 20, 9001, 528, 8, None), ("mid32", 40, [1, 2, 3] * 10 + [20, 0, 7], 50, 4098, 528, 8, "silu"), ("mid32", 8, [33, 1, 0, 64, 2, 90], 100, 9001, 4112, 2, None),
    ("mid64", 3, [100, 0, 301], 300, 2304, 2064, 8, "gelu"), ("mid64", 8, [1400, 0, 0, 0, 100, 0, 0, 0], 300, 1027, 16, 8, None),
    ("mid96", 8, [100, 1, 0, 150, 97, 0, 53], 300, 4099, 528, 8, None),
    ("deep128", 3, [128, 640, 2], 500, 2304, 4112, 8, "silu"), ("deep128", 8, [1, 127, 129, 0, 0, 256, 257, 1], 333, 2304, 1040, 8, None),
    ("tile128", 3, [1000, 1, 499], 500, 4352, 144, 8, "silu"), ("tile128", 40, [150] * 40, 2000, 9001, 144, 4, None),
    ("tile256", 8, [300, 0, 1, 600, 255, 256, 88, 0], 1000, 4099, 528, 8, None), ("tile256", 3, [2000, 4000, 0], 5000, 2304, 144, 8, "gelu"),
    ("tile256", 3, [1, 5998, 1], 3000, 9002, 144, 8, "silu"), ("tile256", 8, [3000, 0, 2, 0, 0, 1480, 1, 1517], 3000, 9001, 144, 4, None),
]


def expected(case):
    f = int8_plans.form(*case[3:6])
    return (f.name, f.ranges > 1, f.quarters)


@pytest.mark.parametrize("case", DENSE)
def test_sizes_take_the_form_that_they_stand_for(case):
    assert expected(case) == case[:3]


def test_all_forms_are_there():
    assert {c[:3] for c in DENSE} >= {(f, False, False) for f in int8_plans.FORMS} | {("mid32", True, False), ("mid64", True, False), ("mid96", True, False), ("deep128", True, False), ("tile256", False, True)}
    for T, N, K, wide in SINGLE:
        assert int8_plans.form(T, N, K).single == (2 if wide else 1)
    for name, E, counts, M, N, K, r, gate in EXPERTS:
        f = int8_plans.form(sum(counts), N, K, E)
        assert f.name == name and not f.single, (name, E, N, K, f)
        assert len(counts) <= E
    assert {c[0] for c in EXPERTS} == set(int8_plans.FORMS)


# ---- on the GPU ----------------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def mq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_06786_amd
    return paper_2502_06786_amd


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def inputs(M, E, N, K, r):
    g = gen(M + 7 * N + 13 * K)
    x = (torch.randn(M, K, generator=g, device="cuda") * torch.exp(2.0 * torch.randn(M, 1, generator=g, device="cuda"))).to(torch.bfloat16)
    codes = torch.randint(0, 1 << r, (E, N, K), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    alpha = torch.exp(torch.randn(E, N, generator=g, device="cuda")) * 0.01
    return x, codes, alpha, 128.0 + 40.0 * torch.randn(E, N, generator=g, device="cuda")


def check(got, tokens, codes, alpha, zero, r, gate, what):
    """against the definition; the 64-bit product of whole numbers is formed on the GPU (exact: sums below 2^53)"""
    codes_x, scale, sums = tokens
    total = codes_x.double().sum(1)
    assert torch.equal(total, sums.double())
    dot = codes_x.double() @ (codes.double() - ref.code_offset(r)).t().contiguous()
    want, bar = ref.outputs(dot.cpu().numpy(), total.cpu().numpy(), scale.cpu().numpy(), alpha.cpu().numpy(), zero.cpu().numpy(), r, gate)
    ref.within(got.cpu().double().numpy(), want, bar, what)


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("case", DENSE)
def test_dense_form(mq, case):
    print(case, flush=True)
    _, _, _, T, N, K, r, gate = case
    x, codes, alpha, zero = inputs(T, 1, N, K, r)
    w = (codes[0], alpha[0], zero[0])
    tokens = mq.mq_quantize_tokens(x)
    n_out = N // 2 if gate else N
    y = torch.full((T + 2, n_out), 3.0, dtype=torch.bfloat16, device="cuda")   # rows before and after are watched
    out = mq.mq_linear_fwd_int8(x, *w, r, gate=gate, Y=y[1:-1]) if (n_out * 2) % 16 == 0 else mq.mq_linear_fwd_int8(x, *w, r, gate=gate, Y=y[:-2])
    assert bool((y[-1] == 3.0).all()) and (out.data_ptr() == y.data_ptr() or bool((y[0] == 3.0).all()))
    check(out, tokens, *w, r, gate, case)
    assert same_bits(mq.mq_linear_fwd_int8_quantized(*tokens, *w, r, gate=gate), out)
    # without room for partial sums, and in other forms: the same bits
    least = torch.empty(mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_FWD_INT8, T, N, K, 1), dtype=torch.uint8, device="cuda")
    assert same_bits(mq.mq_linear_fwd_int8(x, *w, r, gate=gate, ws=least), out)
    for first, n in ((0, 1), (max(0, T - 20), min(20, T))):
        assert same_bits(mq.mq_linear_fwd_int8(x[first:first + n].contiguous(), *w, r, gate=gate), out[first:first + n])


@pytest.mark.gpu
@pytest.mark.parametrize("T,N,K,wide", SINGLE)
@pytest.mark.parametrize("r,gate", [(8, None), (8, "silu"), (3, "gelu")])
def test_single_tokens(mq, T, N, K, wide, r, gate):
    print(T, N, K, r, gate, flush=True)
    N += N % 2 if gate else 0
    x, codes, alpha, zero = inputs(T, 1, N, K, r)
    w = (codes[0], alpha[0], zero[0])
    y = mq.mq_linear_fwd_int8(x, *w, r, gate=gate)
    tokens = mq.mq_quantize_tokens(x)
    check(y, tokens, *w, r, gate, (T, N, K))
    assert same_bits(mq.mq_linear_fwd_int8_quantized(*tokens, *w, r, gate=gate), y)


@pytest.mark.gpu
def test_single_tokens_that_are_special(mq):
    """Zeros, infinities, NaN and the smallest numbers, quantized by the product's workgroups as by the quantizer."""
    from tests.test_gpu_int8 import special_rows
    rows = torch.stack(list(special_rows().values())).to(torch.bfloat16).cuda()
    _, codes, alpha, zero = inputs(1, 1, 40, rows.shape[1], 8)
    w = (codes[0], alpha[0], zero[0])
    whole = mq.mq_linear_fwd_int8_quantized(*mq.mq_quantize_tokens(rows), *w, 8)
    for first in range(0, len(rows), 3):
        part = mq.mq_linear_fwd_int8(rows[first:first + 3].contiguous(), *w, 8)
        want = whole[first:first + 3]
        assert torch.equal(torch.isnan(part), torch.isnan(want)) and torch.equal(torch.nan_to_num(part.float()), torch.nan_to_num(want.float()))


@pytest.mark.gpu
@pytest.mark.parametrize("case", EXPERTS)
def test_experts_form(mq, case):
    print(case[:2], case[3:], flush=True)
    _, E, counts, M, N, K, r, gate = case
    counts = counts + [0] * (E - len(counts))
    T = sum(counts)
    x, codes, alpha, zero = inputs(M, E, N, K, r)
    g = gen(T)
    rows = torch.randint(0, M, (T,), generator=g, device="cuda", dtype=torch.int32)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32).cuda()
    y = mq.mq_experts_fwd_int8(x, offsets, codes, alpha, zero, r, rows=rows, gate=gate)
    tokens = mq.mq_quantize_tokens(x)
    first = 0
    for e, n in enumerate(counts):
        if n:
            at = rows[first:first + n].long()
            check(y[first:first + n], [t[at] for t in tokens], codes[e], alpha[e], zero[e], r, gate, (case, e))
        first += n
    # the same places without a gather
    assert same_bits(mq.mq_experts_fwd_int8(x[rows.long()], offsets, codes, alpha, zero, r, gate=gate), y)


@pytest.mark.gpu
@pytest.mark.parametrize("E,counts,N,K", [(2, [1, 1], 2304, 2064), (8, [0, 0, 3, 0, 0, 0, 1], 520, 4112), (64, [0] * 60 + [1, 0, 2, 1], 2050, 272), (3, [0, 4, 0], 333, 1040),
                                          (8, [1, 0, 0, 1], 18434, 144), (4, [0, 0, 0, 0], 64, 64),
                                          (8, [8], 1027, 1040), (3, [0, 3, 5], 2304, 2064), (64, [0] * 50 + [1, 2, 1, 0, 3], 515, 4112), (8, [1] * 8, 130, 16)])
def test_experts_of_single_tokens(mq, E, counts, N, K):
    counts = counts + [0] * (E - len(counts))
    T = max(1, sum(counts))
    x, codes, alpha, zero = inputs(3, E, N, K, 8)
    rows = (torch.arange(T, dtype=torch.int32) * 2 % 3).cuda()
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32).cuda()
    y = torch.full((T, N), 5.0, dtype=torch.bfloat16, device="cuda")
    mq.mq_experts_fwd_int8(x, offsets, codes, alpha, zero, 8, rows=rows, Y=y)
    tokens = mq.mq_quantize_tokens(x)
    first = 0
    for e, n in enumerate(counts):
        if n:
            check(y[first:first + n], [t[rows[first:first + n].long()] for t in tokens], codes[e], alpha[e], zero[e], 8, None, (E, e))
        first += n
    assert bool((y[first:] == 5.0).all())


@pytest.mark.gpu
def test_gathered_tokens_past_two_gigabytes(mq):
    """They are quantized in the order of the places then."""
    M, K, N, E = 140000, 16384, 48, 3
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([5, 139999, 131071, 131072, 131073, 0, 139999], dtype=torch.int32, device="cuda")
    some, codes, alpha, zero = inputs(7, E, N, K, 8)
    x[rows.long()] = some
    offsets = torch.tensor([0, 3, 3, 7], dtype=torch.int32, device="cuda")
    y = mq.mq_experts_fwd_int8(x, offsets, codes, alpha, zero, 8, rows=rows)
    want = mq.mq_experts_fwd_int8(x[rows.long()], offsets, codes, alpha, zero, 8)
    assert same_bits(y, want)
    for lo, hi, e in ((0, 3, 0), (3, 7, 2)):
        part = mq.mq_linear_fwd_int8(x[rows[lo:hi].long()], codes[e], alpha[e], zero[e], 8)
        assert same_bits(y[lo:hi], part)
