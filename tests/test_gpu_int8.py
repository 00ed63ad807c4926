"""The layer in 8-bit integers on the GPU against its definition: tokens quantized, dense products, products by expert."""
import numpy as np
import pytest
import torch

from tests import int8_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_06786_amd
    return paper_2502_06786_amd


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def rand(seed):
    return torch.Generator().manual_seed(seed)


def tokens(seed, M, K):
    """bf16 on the host, a size of its own for each token"""
    g = rand(seed)
    return (torch.randn(M, K, generator=g) * torch.exp(2.0 * torch.randn(M, 1, generator=g))).to(torch.bfloat16)


def weights(seed, N, K, r):
    g = rand(seed + 1)
    codes = torch.randint(0, 1 << r, (N, K), generator=g, dtype=torch.int32).to(torch.uint8)
    alpha = torch.exp(torch.randn(N, generator=g)) * 0.01
    return codes, alpha, 128.0 + 40.0 * torch.randn(N, generator=g)


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


# ---- tokens ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("M,K,pad", [(1, 16, 0), (3, 48, 0), (65, 256, 8), (5, 4096, 0), (7, 4112, 24), (2, 16384, 0), (3, 16400, 0),
                                     (1, 131072, 0), (300, 1008, 0), (2, 65536, 16), (513, 1024, 0), (4, 1040, 8), (513, 1040, 0), (515, 2048, 8),
                                     (513, 2064, 0), (257, 4112, 0), (259, 16384, 0)])
def test_tokens(mq, M, K, pad):
    x = tokens(M * 7 + K, M, K + pad)
    got = mq.mq_quantize_tokens(x.cuda()[:, :K])
    x = x[:, :K].float().numpy()
    codes, scale, sums = ref.quantize_tokens(x)
    assert np.array_equal(got[0].cpu().numpy(), codes)
    assert np.array_equal(got[1].cpu().numpy(), scale)
    assert np.array_equal(got[2].cpu().numpy(), sums)
    # and the definition in 64 bits: at most half a step and the two fp32 roundings away
    top = np.abs(x.astype(np.float64)).max(axis=1, keepdims=True)
    assert np.all(np.abs(codes - x * 127.0 / top) <= 0.5 + 127.0 * 2.0 ** -22)


def special_rows():
    """name -> one row of 48 values"""
    inf, nan = float("inf"), float("nan")
    g = rand(5)
    r = torch.randn(48, generator=g)
    rows = {"zeros": r * 0, "minus zeros": r * -0.0, "ties": torch.arange(48) - 23.5, "smallest": r * 0 + 2.0 ** -133, "subnormal": r * 2.0 ** -130,
            "at the lift": r * 2.0 ** -101, "largest": r.sign() * 3.38e38, "one value": r * 0, "minus only": -r.abs(), "infinity": r.clone(),
            "minus infinity": r.clone(), "nan": r.clone(), "nan and infinity": r.clone(), "ordinary": r}
    rows["ties"][0] = 127.0
    rows["one value"][47] = -1e-20
    rows["infinity"][3] = inf
    rows["minus infinity"][47] = -inf
    rows["nan"][40] = nan
    rows["nan and infinity"][0], rows["nan and infinity"][1] = nan, inf
    return rows


def test_tokens_special_rows(mq):
    rows = special_rows()
    x = torch.stack(list(rows.values())).to(torch.bfloat16)
    codes, scale, sums = (t.cpu().numpy() for t in mq.mq_quantize_tokens(x.cuda()))
    want = ref.quantize_tokens(x.float().numpy())
    assert np.array_equal(codes, want[0]) and np.array_equal(scale, want[1], equal_nan=True) and np.array_equal(sums, want[2])
    for i, name in enumerate(rows):
        if "infinity" in name or "nan" in name:
            assert np.isnan(scale[i]) and not codes[i].any(), name
        elif "zeros" in name:
            assert scale[i] == 0 and not codes[i].any(), name
        else:
            assert np.abs(codes[i]).max() == 127 and scale[i] > 0, name


# ---- dense -------------------------------------------------------------------------------------------------------------
def check_dense(mq, M, N, K, r, gate, seed=0):
    x = tokens(seed + M + N, M, K)
    codes, alpha, zero = weights(seed + K, N, K, r)
    dev = [t.cuda() for t in (x, codes, alpha, zero)]
    y = mq.mq_linear_fwd_int8(*dev, r, gate=gate)
    cx, s, _ = ref.quantize_tokens(x.float().numpy())
    want, bar = ref.layer(cx, s, codes.numpy(), alpha.numpy(), zero.numpy(), r, gate)
    ref.within(f64(y), want, bar, (M, N, K, r, gate))
    again = mq.mq_linear_fwd_int8_quantized(*mq.mq_quantize_tokens(dev[0]), *dev[1:], r, gate=gate)
    assert same_bits(y, again)
    return dev, y


# tokens around the sizes at which a block or a tile ends
@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 96, 127, 128, 129, 191, 193, 255, 256, 257, 300, 511, 513])
def test_dense_tokens(mq, M):
    check_dense(mq, M, 320, 272, 8 if M % 2 else 4, None)


@pytest.mark.parametrize("N", [1, 2, 3, 7, 8, 15, 16, 17, 63, 64, 65, 127, 129, 130, 255, 256, 257, 383, 511, 515])
@pytest.mark.parametrize("M", [1, 19, 150, 270])
def test_dense_channels(mq, M, N):
    check_dense(mq, M, N, 192, 8, None)


@pytest.mark.parametrize("K", [16, 32, 48, 64, 80, 112, 128, 144, 240, 256, 272, 384, 400, 512, 1008, 2064, 4096, 8208])
@pytest.mark.parametrize("M", [1, 7, 40, 260])
def test_dense_lengths(mq, M, K):
    check_dense(mq, M, 200, K, 8, None)


@pytest.mark.parametrize("r", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("M,gate", [(3, None), (140, "silu"), (300, "gelu")])
def test_dense_bits(mq, r, M, gate):
    check_dense(mq, M, 264, 336, r, gate)


@pytest.mark.parametrize("gate", ["gelu", "silu"])
@pytest.mark.parametrize("M,N,K", [(1, 2, 16), (2, 6, 64), (16, 130, 528), (33, 514, 256), (100, 254, 144), (128, 256, 128), (257, 510, 272)])
def test_dense_gated(mq, M, N, K, gate):
    check_dense(mq, M, N, K, 8, gate)


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (16, 2304, 9216), (61, 1536, 4096), (77, 4096, 2304), (640, 1200, 3584), (1100, 2056, 1040)])
def test_dense_layers(mq, M, N, K):
    check_dense(mq, M, N, K, 8, None)


def test_sums_at_the_end_of_32_bits(mq):
    """127 x -128 and 127 x 127, 131072 times."""
    K = 131072
    x = torch.ones(3, K)
    x[1] = -1.0
    x[2, ::2] = -1.0
    for M in (3, 70):
        x_ = x.repeat(-(-M // 3), 1)[:M].to(torch.bfloat16)
        for code in (0, 255):
            codes = torch.full((40, K), code, dtype=torch.uint8)
            alpha, zero = torch.full((40,), 1e-4), torch.full((40,), 100.0)
            y = mq.mq_linear_fwd_int8(x_.cuda(), codes.cuda(), alpha.cuda(), zero.cuda(), 8)
            cx, s, _ = ref.quantize_tokens(x_.float().numpy())
            want, bar = ref.layer(cx, s, codes.numpy(), alpha.numpy(), zero.numpy(), 8)
            ref.within(f64(y), want, bar, (M, code))


@pytest.mark.parametrize("repeat", [1, 8, 20])
def test_special_tokens_leave_the_others_alone(mq, repeat):
    rows = special_rows()
    x = torch.stack(list(rows.values())).to(torch.bfloat16).repeat(repeat, 1)
    codes, alpha, zero = weights(3, 72, 48, 8)
    dev = [t.cuda() for t in (codes, alpha, zero)]
    y = mq.mq_linear_fwd_int8(x.cuda(), *dev, 8)
    cx, s, _ = ref.quantize_tokens(x.float().numpy())
    with np.errstate(over="ignore", invalid="ignore"):
        want, bar = ref.layer(cx, s, codes.numpy(), alpha.numpy(), zero.numpy(), 8)
    names = list(rows) * repeat
    for i, name in enumerate(names):
        row = f64(y[i])
        if "infinity" in name or "nan" in name:
            assert np.isnan(row).all(), name
        elif "zeros" in name:
            assert not row.any(), name
        elif name == "largest":   # outputs past the largest bf16 number are infinities
            big = np.abs(want[i]) > 3.4e38
            assert np.isinf(row[big]).all()
            ref.within(row[~big], want[i][~big], bar[i][~big], name)
        else:
            ref.within(row, want[i], bar[i], name)


def test_a_token_has_the_same_bits_in_any_call(mq):
    dev, y = check_dense(mq, 600, 1032, 1296, 4, None)
    for part in ([0], [599], range(3), range(40, 56), range(100, 133), range(200, 300), range(7, 300)):
        at = torch.tensor(list(part)).cuda()
        assert same_bits(mq.mq_linear_fwd_int8(dev[0][at], *dev[1:], 4), y[at]), part
    for n in (1, 9, 64, 500):
        part = mq.mq_linear_fwd_int8(dev[0], *[t[:n].contiguous() for t in dev[1:]], 4)
        assert same_bits(part, y[:, :n]), n


def test_sliced_weights(mq):
    """Quantized and sliced by this library: close to what the bf16 forward makes of the same codes."""
    g = rand(9)
    W, x = (torch.randn(256, 512, generator=g) * 0.02).cuda(), torch.randn(64, 512, generator=g).to(torch.bfloat16).cuda()
    Q, alpha, zero = mq.mq_quantize_int8(W)
    for r in (8, 4, 2):
        codes = mq.mq_slice(Q, r)
        y = mq.mq_linear_fwd_int8(x, codes, alpha, zero, r)
        cx, s, _ = ref.quantize_tokens(x.float().cpu().numpy())
        want, bar = ref.layer(cx, s, codes.cpu().numpy(), alpha.cpu().numpy(), zero.cpu().numpy(), r)
        ref.within(f64(y), want, bar, r)
        # a token's rounding is half a step of top / 127 at most, uniform: its share of an output's size is 1/sqrt(12) step / rms of x
        full = mq.mq_linear_fwd_multi(x, Q, alpha, zero, [r])[0]
        step = float(x.float().abs().amax(1).mean()) / 127.0
        assert float((y.float() - full.float()).norm() / full.float().norm()) < 2.0 * step / 12 ** 0.5 + 2.0 ** -8


def test_codes_of_sizes_past_32_bits(mq):
    """Tokens of 2.4 GB, outputs of 5.6 GB."""
    M, K, N = 150000, 16384, 16
    x = tokens(1, 64, K).cuda()
    big = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, 131071, 131072, 131073, M - 1], device="cuda")
    big[at] = x[:6]
    codes, alpha, zero = (t.cuda() for t in weights(2, N, K, 8))
    y = mq.mq_linear_fwd_int8(big, codes, alpha, zero, 8)
    assert same_bits(y[at], mq.mq_linear_fwd_int8(x[:6], codes, alpha, zero, 8))
    del big, y
    M, K, N = 70000, 16, 40008
    x = tokens(4, M, K).cuda()
    codes, alpha, zero = (t.cuda() for t in weights(5, N, K, 8))
    y = mq.mq_linear_fwd_int8(x, codes, alpha, zero, 8)
    at = torch.tensor([0, 26000, 53000, 53674, 53675, 69999], device="cuda")
    assert same_bits(y[at], mq.mq_linear_fwd_int8(x[at], codes, alpha, zero, 8))


# ---- by expert -----------------------------------------------------------------------------------------------------------
def check_experts(mq, counts, M, N, K, r, gate=None, gather=True, spare=0, seed=0):
    """Groups of the given sizes; each expert's part has to have the bits of the dense call."""
    E, T = len(counts), sum(counts) + spare
    g = rand(seed + T)
    x = tokens(seed + N, M if gather else T, K).cuda()
    codes, alpha, zero = (t.cuda() for t in weights(seed + K, E * N, K, r))
    codes, alpha, zero = codes.view(E, N, K), alpha.view(E, N), zero.view(E, N)
    rows = torch.randint(0, x.shape[0], (T,), generator=g, dtype=torch.int32) if gather else torch.arange(T, dtype=torch.int32)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32).cuda()
    if spare:
        rows[-spare:] = -1
    y = torch.full((T, N // 2 if gate else N), 7.0, dtype=torch.bfloat16, device="cuda")
    out = mq.mq_experts_fwd_int8(x, offsets, codes, alpha, zero, r, rows=rows.cuda() if gather else None, gate=gate, Y=y)
    assert out is y
    first = 0
    for e, n in enumerate(counts):
        if n:
            want = mq.mq_linear_fwd_int8(x[rows[first:first + n].long().cuda()], codes[e], alpha[e].clone(), zero[e].clone(), r, gate=gate)
            assert same_bits(y[first:first + n], want), (e, n)
        first += n
    assert bool((y[first:] == 7.0).all())   # places of no expert
    return x, rows, codes, alpha, zero, y


@pytest.mark.parametrize("counts", [[1], [0, 1], [1, 0], [0, 0, 5, 0], [3, 0, 17, 1], [16, 16], [33, 0, 0, 64, 1, 130], [128, 127, 129], [256, 1, 255],
                                    [300], [0] * 63 + [4], [4] + [0] * 63, [1] * 65, [2, 0, 1] * 43, [0] * 64 + [20, 300] + [0] * 62])
def test_experts_groups(mq, counts):
    check_experts(mq, counts, 50, 136, 208, 8)
    check_experts(mq, counts, 50, 136, 208, 4, gather=False)


@pytest.mark.parametrize("N,K,r,gate", [(1, 16, 8, None), (17, 48, 2, None), (65, 144, 8, None), (258, 1040, 3, "silu"), (512, 256, 8, "gelu"), (1000, 528, 8, None)])
def test_experts_sizes(mq, N, K, r, gate):
    check_experts(mq, [5, 0, 70, 1, 150, 0, 9], 80, N, K, r, gate, spare=6)
    check_experts(mq, [1, 0, 2, 1, 0, 0, 3], 7, N, K, r, gate, spare=1)
    check_experts(mq, [500, 0, 270, 600], 700, N, K, r, gate)


def test_experts_against_the_definition(mq):
    counts = [40, 0, 3, 90]
    x, rows, codes, alpha, zero, y = check_experts(mq, counts, 60, 192, 320, 8, "silu")
    first = 0
    for e, n in enumerate(counts):
        part = x[rows[first:first + n].long().cuda()].float().cpu().numpy()
        if n:
            cx, s, _ = ref.quantize_tokens(part)
            want, bar = ref.layer(cx, s, codes[e].cpu().numpy(), alpha[e].cpu().numpy(), zero[e].cpu().numpy(), 8, "silu")
            ref.within(f64(y[first:first + n]), want, bar, e)
        first += n


def test_experts_with_codes_past_32_bits(mq):
    E, N, K = 5, 30000, 32768   # 4.9 GB of codes
    codes = torch.empty(E, N, K, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    for e in range(E):
        codes[e] = torch.randint(0, 256, (1, K), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
        codes[e, -40:] = torch.randint(0, 256, (40, K), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    alpha, zero = torch.full((E, N), 0.01, device="cuda"), torch.full((E, N), 128.0, device="cuda")
    for counts in ([1, 0, 0, 2, 3], [70, 0, 1, 0, 150], [600, 0, 0, 0, 700]):
        T = sum(counts)
        x = tokens(6, T, K).cuda()
        offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32).cuda()
        y = mq.mq_experts_fwd_int8(x, offsets, codes, alpha, zero, 8)
        want = mq.mq_linear_fwd_int8(x[-2:], codes[4, -40:].contiguous(), alpha[4, -40:].contiguous(), zero[4, -40:].contiguous(), 8)
        assert same_bits(y[-2:, -40:], want), counts


@pytest.mark.parametrize("E", [1, 2, 8, 63, 64, 65, 255, 1024])
@pytest.mark.parametrize("M,top", [(0, 2), (1, 1), (1, 4), (31, 2), (64, 1), (1000, 4), (1024, 4), (1025, 4), (5000, 3), (16411, 2)])
def test_route(mq, M, top, E):
    g = rand(M + E)
    ids = torch.randint(0, E, (M, top), generator=g, dtype=torch.int32)
    if E > 4:
        ids[torch.rand(M, top, generator=g) < 0.3] = E // 3   # one is chosen most
    lost = torch.rand(M, top, generator=g)
    ids[lost < 0.05] = -1
    ids[lost > 0.97] = E
    ids[(lost > 0.5) & (lost < 0.51)] = -(1 << 31)
    got = mq.mq_experts_route(ids.cuda(), E)
    for a, b in zip(got, ref.route(ids.numpy(), E)):
        assert np.array_equal(a.cpu().numpy(), b)


@pytest.mark.parametrize("M,top,N", [(1, 1, 8), (1, 2, 1), (3, 4, 2304), (257, 2, 520), (100, 3, 77), (40, 64, 16), (5, 2, 70000)])
def test_combine(mq, M, top, N):
    g = rand(M + N)
    T = M * top
    y = torch.randn(T, N, generator=g).to(torch.bfloat16)
    place = torch.randperm(T, generator=g).to(torch.int32).view(M, top)
    place[torch.rand(M, top, generator=g) < 0.2] = -1
    if M > 2:
        place[1] = -1          # a token with no expert
        place[2, 0] = T        # not a place
    weight = torch.randn(M, top, generator=g)
    out = mq.mq_experts_combine(y.cuda(), place.cuda(), weight.cuda())
    want, bar = ref.combine(f64(y), place.numpy().astype(np.int64), weight.numpy())
    ref.within(f64(out), want, bar)
    if M > 2:
        assert not out[1].any()


def layer_of_experts(mq, x, ids, weight, one, two, r, gate, buffers=None):
    b = buffers or {}
    offsets, rows, place = mq.mq_experts_route(ids, one[0].shape[0], *b.get("route", (None, None, None)), ws=b.get("ws"))
    a = mq.mq_experts_fwd_int8(x, offsets, *one, r, rows=rows, gate=gate, Y=b.get("a"), ws=b.get("ws"))
    y = mq.mq_experts_fwd_int8(a, offsets, *two, r, Y=b.get("y"), ws=b.get("ws"))
    return mq.mq_experts_combine(y, place, weight, out=b.get("out"))


def expert_layer_inputs(M, top, E, d, F, seed=0):
    g = rand(seed)
    x = torch.randn(M, d, generator=g).to(torch.bfloat16).cuda()
    ids = torch.randint(0, E, (M, top), generator=g, dtype=torch.int32).cuda()
    ids[M // 2] = -1
    weight = torch.softmax(torch.randn(M, top, generator=g), 1).cuda()

    def stack(N, K, s):
        c, a, z = weights(s, E * N, K, 8)
        return c.view(E, N, K).cuda(), a.view(E, N).cuda() * 0.1, z.view(E, N).cuda()
    return x, ids, weight, stack(2 * F, d, seed + 1), stack(d, F, seed + 2)


@pytest.mark.parametrize("M", [1, 5, 90])
def test_layer_of_experts(mq, M):
    """All four calls against the definition, token by token; each operator's output is rounded to bf16."""
    d, F, E, top = 96, 128, 6, 2
    x, ids, weight, one, two = expert_layer_inputs(M, top, E, d, F)
    out = layer_of_experts(mq, x, ids, weight, one, two, 8, "gelu")
    n1, n2 = [[t.cpu().numpy() for t in p] for p in (one, two)]
    for m in range(M):
        total = np.zeros((1, d))
        size = 0.0
        for j in range(top):
            e = int(ids[m, j])
            if e < 0:
                continue
            cx, s, _ = ref.quantize_tokens(x[m:m + 1].float().cpu().numpy())
            a, _ = ref.layer(cx, s, n1[0][e], n1[1][e], n1[2][e], 8, "gelu")
            a = torch.tensor(a).to(torch.bfloat16).float().numpy()
            cx, s, _ = ref.quantize_tokens(a)
            y, _ = ref.layer(cx, s, n2[0][e], n2[1][e], n2[2][e], 8)
            total += float(weight[m, j]) * y
            size += np.linalg.norm(y)
        # a value of a that rounds to the other bf16 neighbour may move its code by one step: F/100 of them at once are not expected
        err = np.linalg.norm(f64(out[m:m + 1]) - total)
        assert err <= 2.0 ** -7 * size + 1e-30, (m, err, size)


def test_other_stream_and_graph(mq):
    """The calls run on the current stream, and a graph of them gives the eager result at every replay, with other work in between."""
    M, d, F, E = 40, 256, 384, 8
    x, ids, weight, one, two = expert_layer_inputs(M, 2, E, d, F, 3)
    want = layer_of_experts(mq, x, ids, weight, one, two, 8, "silu")
    lin = mq.mq_linear_fwd_int8(x, one[0][0], one[1][0], one[2][0], 8)
    torch.cuda.synchronize()
    T = ids.numel()
    empty = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda")   # noqa: E731
    need = max(mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_FWD_INT8, T, 2 * F, d, 1), mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_FWD_INT8, T, d, F, 1),
               mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_ROUTE, T, E, 0, 1), mq.mq_workspace_bytes(mq.MQ_OP_LINEAR_FWD_INT8, M, 2 * F, d, 1))
    b = {"route": (empty(E + 1, dtype=torch.int32), empty(T, dtype=torch.int32), empty(M, 2, dtype=torch.int32)), "a": empty(T, F), "y": empty(T, d),
         "out": empty(M, d), "ws": empty(need, dtype=torch.uint8)}
    y = empty(M, 2 * F)
    side = torch.cuda.Stream()

    def work():
        layer_of_experts(mq, x, ids, weight, one, two, 8, "silu", b)
        mq.mq_linear_fwd_int8(x, one[0][0], one[1][0], one[2][0], 8, Y=y, ws=b["ws"])

    with torch.cuda.stream(side):
        work()
    side.synchronize()
    assert same_bits(b["out"], want) and same_bits(y, lin)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        work()
    for k in range(4):
        b["out"].fill_(float("nan"))
        y.fill_(float("nan"))
        b["ws"].fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert same_bits(b["out"], want) and same_bits(y, lin), k
        mq.mq_quantize_tokens(x)
        torch.cuda.synchronize()


def test_two_calls_on_two_streams(mq):
    """Calls on different streams with workspaces of their own do not meet."""
    dev = []
    for seed, (M, N, K) in enumerate([(5, 4096, 2048), (300, 1024, 2048)]):
        x = tokens(seed, M, K).cuda()
        dev.append((x, *[t.cuda() for t in weights(seed, N, K, 8)]))
    want = [mq.mq_linear_fwd_int8(*d, 8) for d in dev]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, d in zip(streams, dev):
            with torch.cuda.stream(s):
                got.append(mq.mq_linear_fwd_int8(*d, 8))
        torch.cuda.synchronize()
        assert all(same_bits(a, b) for a, b in zip(got, want))


def test_binding_refuses(mq):
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    c, a, z = torch.zeros(32, 64, dtype=torch.uint8, device="cuda"), torch.zeros(32, device="cuda"), torch.zeros(32, device="cuda")
    mq.mq_linear_fwd_int8(x, c, a, z, 8)
    with pytest.raises(ValueError):
        mq.mq_linear_fwd_int8(x[:, :48], c, a, z, 8)           # K
    with pytest.raises(ValueError):
        mq.mq_linear_fwd_int8(x, c, a[:16], z, 8)
    with pytest.raises(ValueError):
        mq.mq_linear_fwd_int8(x, c, a, z, 8, gate="relu")
    with pytest.raises(ValueError):
        mq.mq_linear_fwd_int8(x.float(), c, a, z, 8)
    with pytest.raises(ValueError):
        mq.mq_linear_fwd_int8(x, c, a, z, 8, Y=torch.zeros(4, 31, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(mq.MqError):
        mq.mq_linear_fwd_int8(x, c, a, z, 9)
    with pytest.raises(mq.MqError):
        mq.mq_linear_fwd_int8(x, c, a, z, 8, ws=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        mq.mq_quantize_tokens(x.cpu())
    with pytest.raises(ValueError):
        mq.mq_quantize_tokens(x.t())
    with pytest.raises(mq.MqError):
        mq.mq_quantize_tokens(torch.zeros(4, 20, dtype=torch.bfloat16, device="cuda"))
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        mq.mq_experts_fwd_int8(x, off, c.view(1, 32, 64), a, z, 8)   # offsets of two experts
    with pytest.raises(ValueError):
        mq.mq_experts_route(torch.zeros(4, 2, dtype=torch.int64, device="cuda"), 4)
    with pytest.raises(ValueError):
        mq.mq_experts_combine(x, torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, device="cuda"))
