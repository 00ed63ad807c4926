"""The layer in 8-bit integers from its definition: whole numbers as they are, the rest in 64 bits, and how far a correct
implementation may be off."""
import numpy as np


def quantize_tokens(x):
    """x fp32 [M, K] holding bf16 values -> (codes int64, scale fp32, sums int64): the definition's fp32 operations, which are IEEE
    ones, one by one."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        top = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(len(x), np.float32)
        finite = np.isfinite(top)
        lift = np.where(top < np.float32(2.0 ** -100), np.float32(2.0 ** 100), np.float32(1.0)).astype(np.float32)
        per = (np.float32(127.0) / (top * lift)).astype(np.float32)
        codes = np.rint((x * lift[:, None]) * per[:, None])
        codes = np.where((finite & (top > 0))[:, None], codes, 0).astype(np.int64)
        scale = np.where(finite, top / np.float32(127.0), np.float32(np.nan)).astype(np.float32)
    return codes, scale, codes.sum(axis=1)


def act(g, gate):
    with np.errstate(over="ignore"):
        arg = g if gate == "silu" else 2.0 * np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)
        return g / (1.0 + np.exp(-arg)), np.abs(arg)


def code_offset(r):
    """What is taken off a code before the product: the bar below is that of sums of centred codes."""
    return 128.0 if r == 8 else 0.0


def layer(codes_x, scale, codes, alpha, zero, r, gate=None):
    """(outputs in 64 bits, bar): |got - outputs| <= bar element by element."""
    cx = codes_x.astype(np.float64)
    return outputs(cx @ (codes.astype(np.float64) - code_offset(r)).T, cx.sum(axis=1), scale, alpha, zero, r, gate)


def outputs(dot, sums, scale, alpha, zero, r, gate=None):
    """layer() from dot [M, N] = sum over k of token code times (code - code_offset) and sums [M] of the tokens' codes.

    The fp32 steps after the exact sums: dot, sum, zero - offset and five operations on them, each off by 2^-24 of terms that are
    not larger than 2^(8-r) |dot| and (|zero| + 128) |sum|: 8 of those at most.  Then one rounding to bf16 (8 significant bits: half a
    spacing is at most 2^-8 of the value).  With a gate, the errors of both outputs pass through a * u (|act'| <= 1.13), and the
    exponential adds (4 + 2 |argument|) 2^-22 of the value: its argument is off by a few 2^-24 of itself, and an absolute error of the
    argument is a relative one of the result."""
    mult, off = float(1 << (8 - r)), code_offset(r)
    a, z, s = alpha.astype(np.float64), zero.astype(np.float64), scale.astype(np.float64)[:, None]
    sums = np.asarray(sums, np.float64)[:, None]
    y = a * (mult * dot - (z - off) * sums) * s
    err = 8 * 2.0 ** -24 * np.abs(a * s) * (mult * np.abs(dot) + (np.abs(z) + 128.0) * np.abs(sums)) + 2.0 ** -140
    if gate is None:
        return y, err + 2.0 ** -8 * (np.abs(y) + err) + 2.0 ** -134
    g, u, eg, eu = y[:, 0::2], y[:, 1::2], err[:, 0::2], err[:, 1::2]
    v, arg = act(g, gate)
    out = v * u
    err = 1.13 * eg * (np.abs(u) + eu) + np.abs(v) * eu + (4.0 + 2.0 * arg) * 2.0 ** -22 * np.abs(out)
    # (past 2^126 the exponential and its reciprocal leave fp32's range: values below 2^-120 of |g u| may vanish)
    return out, err + 2.0 ** -120 * np.abs(g * u) + 2.0 ** -8 * (np.abs(out) + err) + 2.0 ** -134


def route(ids, E):
    """(offsets, rows, place) of choices ids [M, top]."""
    M, top = ids.shape
    flat = ids.reshape(-1).astype(np.int64)
    bucket = np.where((flat >= 0) & (flat < E), flat, E)
    order = np.argsort(bucket, kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(bucket, minlength=E + 1)[:E])])
    place = np.empty(M * top, np.int64)
    place[order] = np.arange(M * top)
    rows = np.where(np.arange(M * top) < offsets[-1], order // top, -1)
    return offsets, rows, np.where(bucket < E, place, -1).reshape(M, top)


def combine(y, place, weight):
    """(sums in 64 bits, bar): fp32 sums of `top` products, one rounding to bf16."""
    y = np.concatenate([y, np.zeros((1, y.shape[1]))])
    at = np.where((place >= 0) & (place < len(y) - 1), place, len(y) - 1)
    terms = y[at] * weight.astype(np.float64)[..., None]
    out, size = terms.sum(axis=1), np.abs(terms).sum(axis=1)
    err = (place.shape[1] + 1) * 2.0 ** -24 * size
    return out, err + 2.0 ** -8 * (np.abs(out) + err) + 2.0 ** -134


def within(got, want, bar, what=""):
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    none = np.isnan(want)
    assert np.array_equal(np.isnan(got), none), (what, "NaN in other places")
    bad = ~none & ~(np.abs(got - want) <= bar)
    if bad.any():
        at = tuple(int(v) for v in np.argwhere(bad)[0])
        raise AssertionError((what, int(bad.sum()), "of", bad.size, "first at", at, got[at], want[at], "bar", bar[at]))
