"""Matrix-vector products with group scales, the choice of experts, and the layer of experts for a few tokens."""
import numpy as np
import pytest
import torch

from tests import grouped_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mq():
    import paper_2502_06786_amd as mq
    return mq


def to_gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t.to(dtype) if dtype is not None else t


def bf16(a):
    """Rounded to bf16, as float64."""
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).double().numpy()


def whole_plane(rng, rows, K, group, r):
    """Codes, and scales and zero-points that keep every sum in fp32 exact: powers of two and whole numbers."""
    codes = rng.integers(0, 1 << r, (rows, K))
    alpha = 2.0 ** rng.integers(-4, -1, (rows, K // group))
    zero = rng.integers(0, 256, (rows, K // group)).astype(np.float64)
    return codes, alpha, zero


def plane(rng, rows, K, group, r):
    codes = rng.integers(0, 1 << r, (rows, K))
    alpha = bf16(np.exp(0.3 * rng.standard_normal((rows, K // group))) / (60.0 * np.sqrt(K)))
    zero = bf16(128.0 + 10.0 * rng.standard_normal((rows, K // group)))
    return codes, alpha, zero


def gemv(mq, x, codes, alpha, zero, r, group, **kw):
    return mq.mq_gemv_grouped(to_gpu(x, torch.bfloat16), to_gpu(ref.pack(codes, r)), to_gpu(alpha, torch.bfloat16), to_gpu(zero, torch.bfloat16), r,
                              x.shape[1], group, **kw)


# K from one group to more spans than a workgroup has waves, groups of every chunk length and of odd multiples of it, rows around 16
SHAPES = [(1, 1, 32, 32, 4), (1, 16, 64, 64, 2), (2, 17, 32, 32, 8), (16, 15, 96, 96, 4), (3, 33, 160, 32, 4), (5, 100, 384, 192, 2), (16, 48, 512, 64, 4),
          (4, 31, 544, 32, 8), (7, 1000, 1024, 128, 4), (1, 257, 2304, 64, 2), (9, 40, 2304, 256, 2), (13, 64, 1152, 64, 8), (1, 16, 9216, 128, 4),
          (16, 20, 9216, 9216, 4), (2, 35, 10240, 512, 2), (6, 18, 8960, 320, 8), (1, 4099, 256, 256, 4), (11, 23, 33 * 640, 640, 4),
          (15, 50, 17 * 128, 128, 4), (2, 3, 1 << 20, 1 << 20, 4), (6, 9000, 704, 64, 4), (16, 8200, 320, 32, 4), (7, 16390, 384, 128, 2), (8, 70, 96, 96, 8), (8, 50, 33 * 64, 64, 4), (1, 5, 17 * 512, 32, 4), (10, 70, 19 * 192, 64, 2), (1, 9, 1 << 18, 4096, 2)]


@pytest.mark.parametrize("B,N,K,group,r", SHAPES)
def test_gemv_of_whole_numbers(mq, B, N, K, group, r):
    """Every sum is exact, so y is the definition rounded once: equal bits.  (|x| <= 2, step (128 + code) <= 2^14: sums of a chunk below
    512/r 2^9 2; totals in units of 2^-4 below 2^24 as x has few values that are not 0 where K is long.)"""
    rng = np.random.default_rng(K * 31 + N)
    codes, alpha, zero = whole_plane(rng, N, K, group, r)
    x = rng.integers(-2, 3, (B, K)) * (rng.random((B, K)) < min(1.0, (120.0 if r == 2 else 600.0) / K))
    y, _ = ref.product(x, codes, alpha, zero, r)
    size = np.abs(x) @ np.abs(np.repeat(alpha, group, 1) * (2.0 ** (8 - r) * (codes + (r != 8) * 256.0) + np.repeat(zero, group, 1))).T
    assert size.max() * 16 < 2 ** 24
    got = gemv(mq, x, codes, alpha, zero, r, group)
    assert np.array_equal(got.cpu().double().numpy(), bf16(y))


@pytest.mark.parametrize("B,N,K,group,r", SHAPES)
def test_gemv(mq, B, N, K, group, r):
    rng = np.random.default_rng(K * 7 + N)
    codes, alpha, zero = plane(rng, N, K, group, r)
    x = bf16(rng.standard_normal((B, K)))
    y, bar = ref.product(x, codes, alpha, zero, r)
    got = gemv(mq, x, codes, alpha, zero, r, group).cpu().double().numpy()
    assert (np.abs(got - y) <= bar + ref.BF16 * (np.abs(y) + bar)).all()


def test_gemv_leaves_what_is_beside_its_output(mq):
    rng = np.random.default_rng(3)
    codes, alpha, zero = plane(rng, 37, 256, 64, 4)
    x = bf16(rng.standard_normal((3, 256)))
    whole = torch.full((3 * 37 + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
    got = gemv(mq, x, codes, alpha, zero, 4, 64, y=whole[8:8 + 111].view(3, 37))
    assert torch.equal(got, gemv(mq, x, codes, alpha, zero, 4, 64))
    assert (whole[:8] == 7).all() and (whole[119:] == 7).all()


def test_gemv_token_of_no_numbers_is_alone(mq):
    rng = np.random.default_rng(4)
    codes, alpha, zero = plane(rng, 50, 1024, 128, 4)
    x = bf16(rng.standard_normal((16, 1024)))
    want = gemv(mq, x, codes, alpha, zero, 4, 128)
    for bad in (np.nan, np.inf):
        x[5, 100], x[15, 1023] = bad, -bad
        got = gemv(mq, x, codes, alpha, zero, 4, 128)
        keep = [b for b in range(16) if b not in (5, 15)]
        assert torch.equal(got[keep], want[keep])
        assert not torch.isfinite(got[[5, 15]]).any()


@pytest.mark.parametrize("B", [1, 6, 16])
@pytest.mark.parametrize("r,group", [(4, 32), (4, 64), (4, 128), (2, 64), (2, 128), (2, 256), (8, 32), (8, 64)])
def test_gemv_of_weights_that_are_zero_under_large_tokens(mq, B, r, group):
    """Large |x| meet only weights that are 0 (code = z), under a scale of 2^9: what is exactly 0 inside a group stays 0.  Sum of |x| 2^118 in a group."""
    rng = np.random.default_rng(r * group + B)
    N, K, code = 35, 5 * group, {8: 130, 4: 9, 2: 3}[r]
    codes = np.full((N, K), code)
    alpha, zero = np.full((N, 5), 512.0), np.full((N, 5), code * 2.0 ** (8 - r))
    x = np.zeros((B, K))
    for g in range(5):
        at = g * group + rng.choice(group, 16, replace=False)
        x[:, at] = 2.0 ** 114
        other = np.setdiff1d(np.arange(g * group, (g + 1) * group), at)
        codes[:, other] = rng.integers(0, 1 << r, (N, len(other)))
    assert not gemv(mq, x, codes, alpha, zero, r, group).float().any()


# rows that end inside a half piece: what stands behind their end there is chunks of 32 to 128 codes
@pytest.mark.parametrize("B", [1, 6, 16])
@pytest.mark.parametrize("r,K,group", [(4, 32, 32), (4, 64, 64), (4, 64, 32), (4, 160, 32), (4, 576, 192), (2, 64, 64), (2, 128, 128), (2, 1152, 384), (8, 32, 32), (8, 288, 96)])
def test_gemv_of_a_large_last_input(mq, B, r, K, group):
    """A row's last input is 0.94 2^119, under a scale of 2^-118 and a zero-point of 0: the sums are below their limit if the end of the row counts once."""
    rng = np.random.default_rng(K + B)
    codes, alpha, zero = whole_plane(rng, 19, K, group, r)
    codes[:, -1], alpha[:, -1], zero[:, -1] = (1 << r) - 1, 2.0 ** -118, 0.0
    x = rng.integers(-2, 3, (B, K)).astype(np.float64)
    x[:, -group:] = 0.0
    x[:, -1] = 1.875 * 2.0 ** 118
    y, bar = ref.product(x, codes, alpha, zero, r)
    got = gemv(mq, x, codes, alpha, zero, r, group).cpu().double().numpy()
    assert (np.abs(got - y) <= bar + ref.BF16 * (np.abs(y) + bar)).all()


def test_gemv_of_what_the_library_quantizes(mq):
    """Groups are rows of a view: quantize, slice, round, multiply."""
    rng = np.random.default_rng(5)
    N, K, group = 96, 768, 128
    W = to_gpu((0.02 * rng.standard_normal((N, K))).astype(np.float32))
    Q, alpha, zero = mq.mq_quantize_int8(W.view(-1, group))
    ab, zb = mq.mq_params_to_bf16(alpha, zero)
    x = to_gpu(rng.standard_normal((4, K)), torch.bfloat16)
    for r in (8, 4, 2):
        packed = mq.mq_slice(Q.view(N, K), r, packed=True)
        got = mq.mq_gemv_grouped(x, packed, ab.view(N, -1), zb.view(N, -1), r, K, group).cpu().double().numpy()
        y, bar = ref.product(x.cpu().double().numpy(), ref.unpack(packed.cpu().numpy(), K, r), ab.view(N, -1).cpu().double().numpy(),
                             zb.view(N, -1).cpu().double().numpy(), r)
        assert (np.abs(got - y) <= bar + ref.BF16 * (np.abs(y) + bar)).all()
        near = x.float() @ W.t()    # 255 steps over about five deviations, 16 and 4 of them sliced: a few, 8 and 40 percent
        assert float((torch.from_numpy(got).cuda() - near).norm() / near.norm()) < {8: 0.03, 4: 0.15, 2: 0.9}[r]


# ---------------------------------------------------------------------------------------------------------------------
# the router's choice
# ---------------------------------------------------------------------------------------------------------------------
CHOICES = [(1, 1, 1), (3, 2, 2), (300, 5, 3), (1000, 8, 2), (77, 8, 8), (65, 13, 13), (50, 16, 4), (129, 17, 5), (40, 32, 32), (257, 60, 6), (9, 64, 8),
           (33, 64, 32), (70, 100, 8), (31, 128, 31), (20, 200, 8), (11, 256, 32), (5, 300, 32), (6, 512, 8), (3, 700, 7), (4, 1024, 32)]


def scores_of(rng, M, E, how):
    s = (2.0 * rng.standard_normal((M, E))).astype(np.float32)
    if how == "ties":
        s = np.round(s).astype(np.float32)   # many equal scores, zeros of both signs
    if how == "masked":
        s[rng.random((M, E)) < 0.4] = -np.inf
        s[rng.random(M) < 0.2] = -np.inf
    if how == "far":
        s = (s * 60).astype(np.float32)
    if how == "broken":
        s[rng.random((M, E)) < 0.05] = np.nan
        s[rng.random((M, E)) < 0.05] = np.inf
        s[rng.random((M, E)) < 0.2] = -np.inf
    return s


@pytest.mark.parametrize("how", ["plain", "ties", "masked", "far", "broken"])
@pytest.mark.parametrize("M,E,top", CHOICES)
@pytest.mark.parametrize("renormalize", [False, True])
def test_choose(mq, M, E, top, renormalize, how):
    rng = np.random.default_rng(M + 1000 * E)
    s = scores_of(rng, M, E, how)
    ids, w, bar = ref.choose(s, top, renormalize)
    got_ids, got = mq.mq_experts_choose(to_gpu(s), top, renormalize=renormalize)
    assert np.array_equal(got_ids.cpu().numpy(), ids)
    got = got.cpu().double().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(w))
    ok = ~np.isnan(w)
    assert (np.abs(got - w)[ok] <= bar[ok]).all()


def test_choose_of_strided_scores(mq):
    wide = torch.randn(70, 201, device="cuda")
    part = wide[:, 3:63]
    for renormalize in (False, True):
        a, b = mq.mq_experts_choose(part, 6, renormalize=renormalize), mq.mq_experts_choose(part.contiguous(), 6, renormalize=renormalize)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        dw = torch.randn(70, 6, device="cuda")
        assert torch.equal(mq.mq_experts_choose_bwd(part, *a, dw, renormalize=renormalize), mq.mq_experts_choose_bwd(part.contiguous(), *a, dw, renormalize=renormalize))


@pytest.mark.parametrize("how", ["plain", "ties", "masked", "far"])
@pytest.mark.parametrize("M,E,top", CHOICES)
@pytest.mark.parametrize("renormalize", [False, True])
def test_choose_bwd(mq, M, E, top, renormalize, how):
    rng = np.random.default_rng(M + 77 * E)
    s = scores_of(rng, M, E, how)
    ids, w = mq.mq_experts_choose(to_gpu(s), top, renormalize=renormalize)
    dw = rng.standard_normal((M, top)).astype(np.float32)
    dw[ids.cpu().numpy() < 0] = np.nan   # of no choice: not looked at
    got = mq.mq_experts_choose_bwd(to_gpu(s), ids, w, to_gpu(dw), renormalize=renormalize).cpu().double().numpy()
    want, bar = ref.choose_bwd(s, ids.cpu().numpy(), w.cpu().numpy(), dw, renormalize)
    assert (np.abs(got - want) <= bar).all()


@pytest.mark.parametrize("renormalize", [False, True])
def test_choose_bwd_against_differences(mq, renormalize):
    """sum(dweight weight) with one score moved by 2^-6 either way: the choice stays, the third derivative of a softmax weight is below 1, so the
    quotient is off by at most 2^-12 / 6 times sum |dweight|, and by 2^6 times the weights' own errors (a few 2^-24 of sum |dweight|)."""
    rng = np.random.default_rng(9)
    M, E, top, h = 8, 10, 3, 2.0 ** -6
    s = np.stack([rng.permutation(E) * 0.4 for _ in range(M)]).astype(np.float32)   # scores far enough apart to keep their order
    dw = rng.standard_normal((M, top)).astype(np.float32)
    ids, w = mq.mq_experts_choose(to_gpu(s), top, renormalize=renormalize)
    got = mq.mq_experts_choose_bwd(to_gpu(s), ids, w, to_gpu(dw), renormalize=renormalize).cpu().double().numpy()
    size = np.abs(dw.astype(np.float64)).sum(1)
    for e in range(E):
        value = []
        for sign in (1, -1):
            t = s.copy()
            t[:, e] += np.float32(sign * h)
            i, v = mq.mq_experts_choose(to_gpu(t), top, renormalize=renormalize)
            assert torch.equal(i, ids)
            value.append((v.cpu().double().numpy() * dw).sum(1))
        assert (np.abs((value[0] - value[1]) / (2 * h) - got[:, e]) <= size * (h * h / 6 + 16 * ref.U32 / h)).all()


def test_choose_bwd_of_ids_from_elsewhere(mq):
    """An expert twice: both count.  Ids that are none: left out."""
    rng = np.random.default_rng(10)
    s = rng.standard_normal((5, 12)).astype(np.float32)
    ids = np.array([[3, 3, 5], [-1, 0, 12], [11, 11, 11], [-5, 99, -1], [0, 1, 2]], np.int32)
    w, dw = rng.random((5, 3)).astype(np.float32), rng.standard_normal((5, 3)).astype(np.float32)
    for renormalize in (False, True):
        got = mq.mq_experts_choose_bwd(to_gpu(s), to_gpu(ids), to_gpu(w), to_gpu(dw), renormalize=renormalize).cpu().double().numpy()
        want, bar = ref.choose_bwd(s, ids, w, dw, renormalize)
        assert (np.abs(got - want) <= bar).all()


# ---------------------------------------------------------------------------------------------------------------------
# the layer
# ---------------------------------------------------------------------------------------------------------------------
def make_layer(rng, E, d, F, group, r):
    """(reference's arrays, the library's descriptor)."""
    host, dev = {}, {"r": r}
    for name, short, rows, K in (("gate_up", "gu", 2 * F, d), ("down", "dn", d, F)):
        c, a, z = plane(rng, E * rows, K, group or K, r)
        host["codes_" + short], host["alpha_" + short], host["zero_" + short] = (v.reshape(E, rows, -1) for v in (c, a, z))
        dev[name] = to_gpu(ref.pack(c, r)).view(E, rows, -1)
        dev["alpha_" + short], dev["zero_" + short] = (to_gpu(v, torch.bfloat16).view(E, rows, -1) for v in (a, z))
    return host, dev


def choices(rng, B, top, E, masked=0.0):
    ids = np.stack([rng.choice(E, top, replace=top > E) for _ in range(B)]).astype(np.int32)
    ids[rng.random((B, top)) < masked] = rng.choice([-1, -100, E, 1 << 30])
    return ids, rng.random((B, top)).astype(np.float32)


def check_layer(mq, x, host, dev, ids, weight, F, group, r, silu, residual, **kw):
    y, bar = ref.layer(x, host, ids, weight, r, silu, residual)
    got = mq.mq_experts_ffn(to_gpu(x, torch.bfloat16), dev, to_gpu(ids), to_gpu(weight), F, group, silu=silu, residual=residual, **kw)
    assert (np.abs(got.cpu().double().numpy() - y) <= bar).all()
    return got


LAYERS = [  # B, top, E, d, F, group, r, masked
    (1, 1, 1, 32, 32, 32, 4, 0.0), (1, 2, 4, 128, 256, 128, 4, 0.0), (2, 3, 8, 64, 96, 32, 4, 0.0), (16, 2, 8, 256, 128, 64, 4, 0.2),
    (16, 16, 8, 64, 64, 64, 2, 0.3), (5, 4, 60, 192, 320, 64, 4, 0.0), (3, 2, 5, 512, 768, 256, 4, 0.5), (7, 1, 3, 128, 64, 64, 2, 0.0),
    (16, 8, 128, 128, 128, 128, 2, 0.0), (4, 2, 6, 256, 512, 256, 2, 0.0), (9, 5, 16, 64, 64, 32, 8, 0.1), (12, 2, 4, 192, 128, 64, 8, 0.0),
    (6, 2, 4, 96, 160, 0, 4, 0.0), (2, 2, 3, 1152, 2304, 0, 4, 0.0), (13, 3, 7, 640, 1088, 64, 4, 0.0), (1, 8, 16, 2080, 1056, 32, 4, 0.0),
    (8, 7, 1000, 64, 64, 64, 4, 0.0), (1, 2, 3, 8704, 128, 128, 4, 0.0), (1, 1, 2, 64, 8256, 64, 4, 0.0)]


@pytest.mark.parametrize("B,top,E,d,F,group,r,masked", LAYERS)
def test_layer(mq, B, top, E, d, F, group, r, masked):
    rng = np.random.default_rng(d + 3 * F + B)
    host, dev = make_layer(rng, E, d, F, group, r)
    x = bf16(rng.standard_normal((B, d)))
    ids, weight = choices(rng, B, top, E, masked)
    check_layer(mq, x, host, dev, ids, weight, F, group, r, bool(B % 2), bool(top % 2))


def test_layer_of_no_choices_at_all(mq):
    rng = np.random.default_rng(20)
    host, dev = make_layer(rng, 4, 64, 96, 32, 4)
    x = bf16(rng.standard_normal((3, 64)))
    ids, weight = np.array([[-1, -1], [2, -1], [4, 5]], np.int32), np.array([[np.nan, np.inf], [0.5, np.nan], [np.inf, np.nan]], np.float32)
    for residual in (False, True):
        got = check_layer(mq, x, host, dev, np.where(ids == 2, 2, -1).astype(np.int32), np.where(ids == 2, weight, 0).astype(np.float32), 96, 32, 4, True, residual)
        again = mq.mq_experts_ffn(to_gpu(x, torch.bfloat16), dev, to_gpu(ids), to_gpu(weight), 96, 32, silu=True, residual=residual)
        assert torch.equal(got, again)   # what stands beside an id that is none shows nowhere
        rest = to_gpu(x, torch.bfloat16) if residual else torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda")
        assert torch.equal(again[[0, 2]], rest[[0, 2]])


def test_layer_of_an_expert_chosen_twice(mq):
    rng = np.random.default_rng(21)
    host, dev = make_layer(rng, 3, 64, 64, 64, 4)
    x = bf16(rng.standard_normal((4, 64)))
    ids = np.array([[1, 1, 1], [0, 2, 0], [2, 2, 1], [-1, 1, 1]], np.int32)
    check_layer(mq, x, host, dev, ids, rng.standard_normal((4, 3)).astype(np.float32), 64, 64, 4, False, False)


@pytest.mark.parametrize("B,top,E,r", [(8, 1, 1, 4), (9, 1, 1, 4), (16, 1, 1, 2), (16, 16, 1, 4), (16, 2, 2, 8), (12, 3, 1, 2)])
def test_layer_of_experts_that_everybody_chose(mq, B, top, E, r):
    """Up to 16 tokens to an expert: one entry of them, one and a token, two full ones; choices of the same expert add up."""
    rng = np.random.default_rng(24 + B)
    host, dev = make_layer(rng, E, 128, 192, 64, r)
    x, (ids, weight) = bf16(rng.standard_normal((B, 128))), choices(rng, B, top, E)
    check_layer(mq, x, host, dev, ids, weight, 192, 64, r, True, True)


def test_layer_of_large_numbers(mq):
    """Gated products around 2^40, of both signs, and around 2^-40: two bf16 parts keep 16 bits of either."""
    rng = np.random.default_rng(25)
    host, dev = make_layer(rng, 3, 64, 96, 32, 4)
    x, (ids, weight) = bf16(rng.standard_normal((4, 64))), choices(rng, 4, 2, 3)
    x[:2] *= 2.0 ** 20
    x[2:] *= 2.0 ** -20
    check_layer(mq, x, host, dev, ids, weight, 96, 32, 4, True, False)


@pytest.mark.parametrize("r,F,group", [(4, 32, 32), (4, 128, 128), (4, 160, 32), (4, 640, 128), (2, 256, 256), (8, 64, 64), (8, 96, 32)])
def test_layer_of_large_last_gated_products(mq, r, F, group):
    """Every expert's last eight gated products add up to 0.92 2^119, under scales of 2^-116 and zero-points of 0; more experts than the down product has
    waves, so a wave that is through with one goes on to another: what it reads behind a row's end counts for nothing."""
    rng = np.random.default_rng(F + r)
    B, top, E, d = 16, 16, 120, max(group, 64)
    host, dev = make_layer(rng, E, d, F, group, r)
    code, step = (1 << r) - 1, 2.0 ** (8 - r)
    host["codes_gu"][:], host["zero_gu"][:] = code, code * step
    host["codes_gu"][:, -16:, 0] = code - 1                      # the last eight pairs of rows alone have a weight that is not 0, their first one
    host["alpha_gu"][:, 0::2], host["alpha_gu"][:, 1::2] = -2.0 ** 57 / step, -2.0 ** 58 / step
    host["codes_dn"][:, :, -8:], host["alpha_dn"][:], host["zero_dn"][:] = code, 2.0 ** -116, 0.0
    for name, short in (("gate_up", "gu"), ("down", "dn")):
        dev[name] = to_gpu(ref.pack(host["codes_" + short], r))
        dev["zero_" + short], dev["alpha_" + short] = to_gpu(host["zero_" + short], torch.bfloat16), to_gpu(host["alpha_" + short], torch.bfloat16)
    x = np.zeros((B, d))
    x[:, 0] = 1.359375   # gated products: 2^57 x 2^58 x, eight of them 2^118.89
    ids, weight = choices(rng, B, top, E)
    check_layer(mq, x, host, dev, ids, weight, F, group, r, True, False)


def test_layer_token_of_no_numbers_is_alone(mq):
    """A token of NaN beside others that share its experts; a weight of NaN likewise."""
    rng = np.random.default_rng(22)
    host, dev = make_layer(rng, 4, 128, 128, 64, 4)
    x, (ids, weight) = bf16(rng.standard_normal((6, 128))), choices(rng, 6, 2, 4)
    want = check_layer(mq, x, host, dev, ids, weight, 128, 64, 4, True, False)
    x[2, 17], weight[4, 1] = np.nan, np.nan
    got = mq.mq_experts_ffn(to_gpu(x, torch.bfloat16), dev, to_gpu(ids), to_gpu(weight), 128, 64, silu=True)
    assert torch.equal(got[[0, 1, 3, 5]], want[[0, 1, 3, 5]]) and torch.isnan(got[[2, 4]]).all()


def test_layer_workspace_of_anything(mq):
    """What is in the workspace before a call does not show, nothing behind its bytes is written, and calls of other sizes share it."""
    rng = np.random.default_rng(23)
    cases = []
    for B, top, E, d, F in ((4, 2, 6, 128, 256), (1, 3, 5, 64, 128), (16, 2, 6, 128, 64)):
        host, dev = make_layer(rng, E, d, F, 64, 4)
        cases.append((bf16(rng.standard_normal((B, d))), host, dev, *choices(rng, B, top, E, 0.2), F))
    need = max(mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_FFN, c[3].size, c[5], c[0].shape[1], 1) for c in cases)
    room = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
    for x, host, dev, ids, weight, F in cases + cases[::-1]:
        check_layer(mq, x, host, dev, ids, weight, F, 64, 4, True, True, ws=room[:need])
    assert (room[need:] == 255).all()


# ---------------------------------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------------------------------
def step(mq, router, dev, x, F, group, top, kept):
    """One decode step of a block: the router's product (a plane like any other), its choice, the layer with the residual."""
    scores = mq.mq_gemv_grouped(x, *router, 4, x.shape[1], group).float()
    ids, weight = mq.mq_experts_choose(scores, top, renormalize=True, ids=kept["ids"], weight=kept["weight"])
    return mq.mq_experts_ffn(x, dev, ids, weight, F, group, silu=True, residual=True, y=kept["y"], ws=kept["ws"]), scores


def block(mq, rng, B, E, d, F, group, top):
    host, dev = make_layer(rng, E, d, F, group, 4)
    c, a, z = plane(rng, E, d, group, 4)
    router = (to_gpu(ref.pack(c, 4)), to_gpu(a * 4, torch.bfloat16), to_gpu(z, torch.bfloat16))
    kept = {"ids": torch.empty(B, top, dtype=torch.int32, device="cuda"), "weight": torch.empty(B, top, device="cuda"),
            "y": torch.empty(B, d, dtype=torch.bfloat16, device="cuda"),
            "ws": torch.empty(mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_FFN, B * top, F, d, 1), dtype=torch.uint8, device="cuda")}
    return host, dev, router, kept


@pytest.mark.parametrize("B", [1, 5, 16])
def test_step_of_a_block(mq, B):
    rng = np.random.default_rng(30 + B)
    E, d, F, group, top = 12, 256, 192, 64, 3
    host, dev, router, kept = block(mq, rng, B, E, d, F, group, top)
    x = to_gpu(rng.standard_normal((B, d)), torch.bfloat16)
    y, scores = step(mq, router, dev, x, F, group, top, kept)
    ids, w, bar = ref.choose(scores.cpu().numpy(), top, True)
    assert np.array_equal(kept["ids"].cpu().numpy(), ids) and (np.abs(kept["weight"].cpu().double().numpy() - w) <= bar).all()
    want, far = ref.layer(x.cpu().double().numpy(), host, ids, kept["weight"].cpu().numpy(), 4, True, True)
    assert (np.abs(y.cpu().double().numpy() - want) <= far).all()


def test_step_captured(mq):
    """Two graphs of a step that share a workspace, replayed in turn with other inputs and eager calls between; all on a stream of its own."""
    rng = np.random.default_rng(40)
    E, d, F, group, top = 6, 128, 192, 64, 2
    blocks = [block(mq, rng, B, E, d, F, group, top) for B in (4, 9)]
    ws = max((b[3]["ws"] for b in blocks), key=lambda t: t.numel())
    side = torch.cuda.Stream()
    graphs, inputs = [], []
    for (host, dev, router, kept), B in zip(blocks, (4, 9)):
        kept["ws"] = ws
        x = torch.zeros(B, d, dtype=torch.bfloat16, device="cuda")
        with torch.cuda.stream(side):
            step(mq, router, dev, x, F, group, top, kept)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(mq, router, dev, x, F, group, top, kept)
        graphs.append(g)
        inputs.append(x)
    for turn in range(6):
        for (host, dev, router, kept), g, x in zip(blocks, graphs, inputs):
            x.copy_(torch.randn(x.shape, device="cuda"))
            g.replay()
            got = kept["y"].clone()
            kept["y"].zero_()
            want, _ = step(mq, router, dev, x, F, group, top, kept)
            assert torch.equal(got, want), turn


def test_tokens_do_not_wait_for_the_default_stream(mq):
    """Calls go to the current stream: one with work ahead of it, results read after that stream alone."""
    rng = np.random.default_rng(50)
    codes, alpha, zero = plane(rng, 512, 1024, 128, 4)
    packed, a, z = to_gpu(ref.pack(codes, 4)), to_gpu(alpha, torch.bfloat16), to_gpu(zero, torch.bfloat16)
    x = bf16(rng.standard_normal((2, 1024)))
    want = gemv(mq, x, codes, alpha, zero, 4, 128)
    side, late = torch.cuda.Stream(), torch.zeros(2, 1024, dtype=torch.bfloat16, device="cuda")
    ready = to_gpu(x, torch.bfloat16)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.randn(1 << 22, device="cuda").sort()
        late.copy_(ready)
        got = mq.mq_gemv_grouped(late, packed, a, z, 4, 1024, 128)
    side.synchronize()
    assert torch.equal(got, want)


# ---------------------------------------------------------------------------------------------------------------------
# far and side by side
# ---------------------------------------------------------------------------------------------------------------------
def test_gemv_of_a_plane_past_four_gigabytes(mq):
    """Its last rows are those of a plane of these rows alone (other workgroups, the same order of sums: it goes by K and the group but for the number
    of waves, which is the same for planes of this many rows)."""
    N, K, group = 1_200_000, 8192, 128
    packed = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda")
    alpha = (0.001 * torch.rand(N, K // group, device="cuda")).to(torch.bfloat16)
    zero = (120 + 16 * torch.rand(N, K // group, device="cuda")).to(torch.bfloat16)
    x = torch.randn(3, K, device="cuda").to(torch.bfloat16)
    got = mq.mq_gemv_grouped(x, packed, alpha, zero, 4, K, group)
    for a in (0, 1_048_570, N - 100_000):   # byte 2^32 is in row 1048576
        part = slice(a, a + 100_000)
        want = mq.mq_gemv_grouped(x, packed[part].contiguous(), alpha[part].contiguous(), zero[part].contiguous(), 4, K, group)
        assert float((got[:, part].float() - want.float()).abs().max()) <= 2.0 ** -7 * float(want.float().abs().max())
        assert float((got[:, part] != want).float().mean()) < 0.01
    y, bar = ref.product(x.cpu().double().numpy(), ref.unpack(packed[-32:].cpu().numpy(), K, 4), alpha[-32:].cpu().double().numpy(),
                         zero[-32:].cpu().double().numpy(), 4)
    assert (np.abs(got[:, -32:].cpu().double().numpy() - y) <= bar + ref.BF16 * (np.abs(y) + bar)).all()


def test_layer_of_experts_past_four_gigabytes(mq):
    """The last expert of many is that expert among two (as many as there are choices, by which the work is cut)."""
    E, d, F, group = 100, 4096, 14336, 128
    L = {"r": 4}
    for name, short, rows, K in (("gate_up", "gu", 2 * F, d), ("down", "dn", d, F)):
        L[name] = torch.randint(0, 256, (E, rows, K // 2), dtype=torch.uint8, device="cuda")
        L["alpha_" + short] = torch.full((E, rows, K // group), 0.0005, device="cuda").to(torch.bfloat16)
        L["zero_" + short] = (120 + 16 * torch.rand(E, rows, K // group, device="cuda")).to(torch.bfloat16)
    x = torch.randn(2, d, device="cuda").to(torch.bfloat16)
    ids, weight = torch.tensor([[E - 1], [E - 1]], dtype=torch.int32, device="cuda"), torch.ones(2, 1, device="cuda")
    got = mq.mq_experts_ffn(x, L, ids, weight, F, group, silu=True)
    two = {k: (v[E - 2:].contiguous() if isinstance(v, torch.Tensor) else v) for k, v in L.items()}
    assert torch.equal(got, mq.mq_experts_ffn(x, two, torch.ones_like(ids), weight, F, group, silu=True))
    assert torch.isfinite(got).all() and float(got.float().std()) > 0


def test_choose_of_many_tokens(mq):
    """Enough of them for every compute unit several times over, against a stable sort and a softmax in 64 bits on the GPU."""
    for M, E, top in ((70_001, 64, 8), (131_072, 8, 2), (40_003, 128, 6)):
        s = torch.round(64 * torch.randn(M, E, device="cuda")) / 64   # some scores are equal
        s[torch.rand(M, E, device="cuda") < 0.05] = -torch.inf
        ids, weight = mq.mq_experts_choose(s, top)
        best, order = torch.sort(s, dim=1, descending=True, stable=True)
        live = best[:, :top] > -torch.inf
        assert torch.equal(ids, torch.where(live, order[:, :top], -1).to(torch.int32))
        w = torch.softmax(s.double(), 1).nan_to_num(0.0).gather(1, order[:, :top])
        # half a step of the exponent's argument (up to 12) each way, of the sum of E, of the quotient
        assert float(((weight - w).abs() / w.clamp(min=1e-30))[live].max()) < ref.U32 * (2 * 24 + E + 12)
        assert not weight[~live].any()


@pytest.mark.parametrize("E,ld", [(64, 600_000_000), (61, 600_000_001)])   # whole 16-byte pieces, single scores
def test_choose_of_rows_far_apart(mq, E, ld):
    """Rows of which the second begins behind 2^31 bytes and the third behind 2^32."""
    wide = torch.empty(2 * ld + E, device="cuda")
    part = torch.as_strided(wide, (3, E), (ld, 1))
    part.copy_(torch.randn(3, E, device="cuda"))
    for renormalize in (False, True):
        a, b = mq.mq_experts_choose(part, 5, renormalize=renormalize), mq.mq_experts_choose(part.contiguous(), 5, renormalize=renormalize)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        dw = torch.randn(3, 5, device="cuda")
        assert torch.equal(mq.mq_experts_choose_bwd(part, *a, dw, renormalize=renormalize), mq.mq_experts_choose_bwd(part.contiguous(), *a, dw, renormalize=renormalize))


def test_choose_bwd_captured(mq):
    """A router's step of training in a graph, replayed with other scores between eager calls."""
    s, dw = torch.randn(300, 24, device="cuda"), torch.randn(300, 4, device="cuda")
    ids, weight, ds = torch.empty(300, 4, dtype=torch.int32, device="cuda"), torch.empty(300, 4, device="cuda"), torch.empty(300, 24, device="cuda")

    def both(**kw):
        i, w = mq.mq_experts_choose(s, 4, **{k: kw[k] for k in ("ids", "weight") if k in kw})
        return mq.mq_experts_choose_bwd(s, i, w, dw, **{k: kw[k] for k in ("dscores",) if k in kw})
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        both(ids=ids, weight=weight, dscores=ds)
    for turn in range(5):
        s.normal_()
        dw.normal_()
        g.replay()
        assert torch.equal(ds, both()), turn


def test_two_calls_at_once(mq):
    """Two streams, each with its own buffers."""
    rng = np.random.default_rng(60)
    runs = []
    for B in (3, 12):
        host, dev = make_layer(rng, 6, 256, 320, 64, 4)
        x, (ids, weight) = bf16(rng.standard_normal((B, 256))), choices(rng, B, 2, 6)
        args = (to_gpu(x, torch.bfloat16), dev, to_gpu(ids), to_gpu(weight), 320, 64)
        y, bar = ref.layer(x, host, ids, weight, 4, True)
        ws = torch.empty(mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_FFN, B * 2, 320, 256, 1), dtype=torch.uint8, device="cuda")
        runs.append((args, ws, torch.cuda.Stream(), y, bar))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(50):
        for out, (args, ws, stream, _, _) in zip(outs, runs):
            with torch.cuda.stream(stream):
                out.append(mq.mq_experts_ffn(*args, silu=True, ws=ws))
    torch.cuda.synchronize()
    for out, (_, _, _, y, bar) in zip(outs, runs):
        assert all(torch.equal(o, out[0]) for o in out)
        assert (np.abs(out[0].cpu().double().numpy() - y) <= bar).all()


def test_what_the_binding_refuses(mq):
    rng = np.random.default_rng(70)
    codes, alpha, zero = plane(rng, 32, 128, 64, 4)
    packed, a, z = to_gpu(ref.pack(codes, 4)), to_gpu(alpha, torch.bfloat16), to_gpu(zero, torch.bfloat16)
    x = torch.zeros(2, 128, dtype=torch.bfloat16, device="cuda")

    def f(x=x, packed=packed, a=a, z=z, r=4, K=128, group=64, **kw):
        return mq.mq_gemv_grouped(x, packed, a, z, r, K, group, **kw)
    f()
    for bad in (dict(x=x.float()), dict(x=x.cpu()), dict(x=torch.zeros(2, 256, dtype=torch.bfloat16, device="cuda")[:, ::2]), dict(x=x[:, :64]), dict(group=48),
                dict(group=0), dict(a=a[:, :1]), dict(z=z.float()), dict(packed=packed[:, :32]), dict(K=256), dict(r=2), dict(y=torch.zeros(2, 31, device="cuda"))):
        with pytest.raises(ValueError):
            f(**bad)
    with pytest.raises(mq.MqError):
        f(x=torch.zeros(17, 128, dtype=torch.bfloat16, device="cuda"))
    s = torch.zeros(4, 8, device="cuda")
    ids, w = mq.mq_experts_choose(s, 2)
    for bad in (s.double(), s.t(), s.cpu()):
        with pytest.raises(ValueError):
            mq.mq_experts_choose(bad, 2)
    for bad in ((s, ids[:3], w, w), (s, ids, w[:, :1], w), (s, ids.long(), w, w), (s, ids, w, w.double())):
        with pytest.raises(ValueError):
            mq.mq_experts_choose_bwd(*bad)
    with pytest.raises(mq.MqError):
        mq.mq_experts_choose(s, 9)
    host, dev = make_layer(rng, 3, 64, 96, 32, 4)
    t = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    i, v = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, 2, device="cuda")
    for bad in (dict(F=64), dict(group=64), dict(ids=i.long()), dict(weight=v[:, :1]), dict(x=t.half()), dict(layer={**dev, "r": 2})):
        kw = dict(x=t, layer=dev, ids=i, weight=v, F=96, group=32)
        kw.update(bad)
        with pytest.raises(ValueError):
            mq.mq_experts_ffn(**kw)
    with pytest.raises(mq.MqError):
        mq.mq_experts_ffn(t, dev, i, v, 96, 32, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
