"""Products with group scales, the choice of experts and the layer of experts for a few tokens from their definitions in 64 bits, and how
far a correct implementation may be off."""
import numpy as np
import torch

U32 = 2.0 ** -24   # half a step of fp32, relative
BF16 = 2.0 ** -8   # half a step of bf16, relative


def unpack(packed, K, r):
    """[..., K*r/8] bytes -> [..., K] codes."""
    bits = np.unpackbits(packed[..., None], axis=-1, bitorder="little").reshape(*packed.shape[:-1], K, r)
    return (bits.astype(np.int64) << np.arange(r)).sum(-1)


def pack(codes, r):
    bits = (codes[..., None] >> np.arange(r) & 1).astype(np.uint8)
    return np.packbits(bits.reshape(*codes.shape[:-1], -1), axis=-1, bitorder="little")


def product(x, codes, alpha, zero, r):
    """x [B, K], codes [N, K], alpha, zero [N, groups] -> (y [B, N], bar before y is rounded).

    The bar: inside a chunk of at most 512 / r codes the matrix core adds products of (128 + code) or code and x, and x alone, one rounding
    per addition at most, each of half a step of a partial sum that is at most the sum of the magnitudes; a chunk's two sums are scaled
    (three roundings, two more for the factors) and added to the row's total, as many times as there are chunks; waves' totals meet in at
    most 16 more additions."""
    x, codes, alpha, zero = (np.asarray(v, np.float64) for v in (x, codes, alpha, zero))
    K = x.shape[1]
    group = K // alpha.shape[1]
    step, offset = 2.0 ** (8 - r), 0.0 if r == 8 else 128.0
    a, z = np.repeat(alpha, group, 1), np.repeat(zero, group, 1)
    y = x @ (a * (step * codes - z)).T
    size = np.abs(x) @ (np.abs(a) * (step * (codes + offset) + np.abs(z) + step * offset)).T
    chunk = min(group, 512 // r)
    return y, U32 * (chunk + K / chunk + 32) * size


def act(g, silu):
    with np.errstate(over="ignore"):
        t = g if silu else 2.0 * np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)
        return g / (1.0 + np.exp(-t))


def layer(x, L, ids, weight, r, silu, residual=False):
    """L: codes_gu [E, 2F, d], alpha_gu, zero_gu [E, 2F, .], codes_dn [E, d, F], alpha_dn, zero_dn -> (y [B, d], bar with y's rounding)."""
    x, weight = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    E, d = L["codes_dn"].shape[:2]
    y, bar = np.zeros((len(x), d)), np.zeros((len(x), d))
    for b in range(len(x)):
        for j in range(ids.shape[1]):
            e = ids[b, j]
            if not 0 <= e < E:
                continue
            h, dh = product(x[b:b + 1], L["codes_gu"][e], L["alpha_gu"][e], L["zero_gu"][e], r)
            g, u, dg, du = h[:, 0::2], h[:, 1::2], dh[:, 0::2], dh[:, 1::2]
            a = act(g, silu) * u
            # the activation's slope is at most 1.13; its hardware exponential and quotient are good to 2^-20 of a value whose exponent is
            # at most |2.3 (g + 0.045 g^3)| + 1 (an error of the exponent's argument, half a fp32 step each way); two bf16 parts hold 2^-16
            t = np.abs(2.3 * (g + 0.045 * g ** 3)) + 1.0
            da = 1.2 * dg * np.abs(u) + (np.abs(act(g, silu)) + 1.2 * dg) * du + np.abs(a) * (2.0 ** -16 + 2.0 ** -20 + 4 * U32 * t)
            o, do = product(a, L["codes_dn"][e], L["alpha_dn"][e], L["zero_dn"][e], r)
            w = np.abs(np.repeat(np.asarray(L["alpha_dn"][e], np.float64), a.shape[1] // L["alpha_dn"].shape[2], 1)
                       * (2.0 ** (8 - r) * L["codes_dn"][e] - np.repeat(np.asarray(L["zero_dn"][e], np.float64), a.shape[1] // L["alpha_dn"].shape[2], 1)))
            y[b] += weight[b, j] * o[0]
            bar[b] += np.abs(weight[b, j]) * (do[0] * 1.01 + (da @ w.T)[0] + 40 * U32 * np.abs(o[0]))
    if residual:
        y = y + x
    return y, bar + BF16 * (np.abs(y) + bar)


def product_on(x, packed, alpha, zero, r):
    """`product` on tensors of any device, codes packed."""
    x, alpha, zero = x.double(), alpha.double(), zero.double()
    rows, groups = alpha.shape
    group, step, offset = x.shape[1] // groups, 2.0 ** (8 - r), 0.0 if r == 8 else 128.0
    codes = torch.stack([(packed >> (r * i)) & ((1 << r) - 1) for i in range(8 // r)], -1).view(rows, groups, group)
    w = alpha[..., None] * (step * codes.double() - zero[..., None])
    size = alpha.abs()[..., None] * (step * (codes.double() + offset) + zero.abs()[..., None] + step * offset)
    chunk = min(group, 512 // r)
    return x @ w.view(rows, -1).t(), U32 * (chunk + x.shape[1] / chunk + 32) * (x.abs() @ size.view(rows, -1).t())


def layer_on(x, L, ids, weight, r, silu, residual=False):
    """`layer` on tensors of any device: packed_gu [E, 2F, d r / 8] and so on; an expert with all its tokens at a time."""
    x, weight = x.double(), weight.double()
    y, bar = torch.zeros_like(x), torch.zeros_like(x)
    for e in range(L["packed_dn"].shape[0]):
        token, choice = (ids == e).nonzero(as_tuple=True)
        if not token.numel():
            continue
        h, dh = product_on(x[token], L["packed_gu"][e], L["alpha_gu"][e], L["zero_gu"][e], r)
        g, u, dg, du = h[:, 0::2], h[:, 1::2], dh[:, 0::2], dh[:, 1::2]
        act = g * torch.sigmoid(g if silu else 2.0 * (2.0 / np.pi) ** 0.5 * (g + 0.044715 * g ** 3))
        a, t = act * u, (2.3 * (g + 0.045 * g ** 3)).abs() + 1.0   # (bounds as in `layer`)
        da = 1.2 * dg * u.abs() + (act.abs() + 1.2 * dg) * du + a.abs() * (2.0 ** -16 + 2.0 ** -20 + 4 * U32 * t)
        o, do = product_on(a, L["packed_dn"][e], L["alpha_dn"][e], L["zero_dn"][e], r)
        w = product_on(torch.eye(a.shape[1], dtype=torch.float64, device=x.device), L["packed_dn"][e], L["alpha_dn"][e], L["zero_dn"][e], r)[0]
        by = weight[token, choice][:, None]
        y.index_add_(0, token, by * o)
        bar.index_add_(0, token, by.abs() * (do * 1.01 + da @ w.abs() + 40 * U32 * o.abs()))
    if residual:
        y = y + x
    return y, bar + BF16 * (y.abs() + bar)


def choose(scores, top, renormalize):
    """scores fp32 [M, E] -> (ids, weight in 64 bits, bar)."""
    s = np.asarray(scores, np.float64)
    M, E = s.shape
    ids, w, bar = np.full((M, top), -1), np.zeros((M, top)), np.zeros((M, top))
    for m in range(M):
        key = np.where(np.isnan(s[m]), np.inf, s[m])
        order = np.argsort(-key, kind="stable")[:top]
        live = key[order] > -np.inf
        ids[m] = np.where(live, order, -1)
        if not live.any():
            continue
        with np.errstate(invalid="ignore"):
            gap = key - key.max()   # inf - inf is no number: so are all weights
            e = np.exp(gap)
        total = e[order[live]].sum() if renormalize else e.sum()
        if np.isnan(e).any():
            total = np.nan
        w[m] = np.where(live, e[order] / total, 0.0)
        # difference and exponential: half a step of the exponent's argument, and two steps; the sum of E of them; the quotient
        with np.errstate(invalid="ignore"):
            bar[m] = np.where(live, w[m] * U32 * (2 * np.abs(gap[order]) + 2 * np.abs(np.where(e > 0, gap * e, 0)).sum() / total + E + 12) + 2.0 ** -126, 0.0)
    return ids, w, bar


def choose_bwd(scores, ids, weight, dweight, renormalize):
    """(dscores [M, E] in 64 bits, bar)."""
    s, weight, dweight = (np.asarray(v, np.float64) for v in (scores, weight, dweight))
    M, E = s.shape
    out, bar = np.zeros((M, E)), np.zeros((M, E))
    top = ids.shape[1]
    for m in range(M):
        live = [j for j in range(top) if 0 <= ids[m, j] < E]
        mean = sum(weight[m, j] * dweight[m, j] for j in live)
        size = sum(abs(weight[m, j] * dweight[m, j]) for j in live)
        up, most = np.zeros(E), np.zeros(E)
        for j in live:
            up[ids[m, j]] += weight[m, j] * (dweight[m, j] - mean) if renormalize else dweight[m, j]
            most[ids[m, j]] += abs(weight[m, j]) * (abs(dweight[m, j]) + size) if renormalize else abs(dweight[m, j])
        if renormalize:
            # below 2^-126 steps of fp32 are no longer relative: 2^-149 each, or the value itself where such numbers count as zero
            out[m], bar[m] = up, U32 * (top + 8) * most + 2.0 ** -126
            continue
        peak = s[m].max()
        e = np.exp(s[m] - peak) if peak > -np.inf else np.zeros(E)
        p = e / e.sum() if e.sum() > 0 else e
        gap = peak - np.where(e > 0, s[m], peak) if peak > -np.inf else np.zeros(E)
        out[m] = p * (up - mean)
        bar[m] = U32 * (p * (top + 8) * (most + size) + p * np.abs(up - mean) * (2 * gap + 2 * (p * gap).sum() + E + 16)) + 2.0 ** -126
    return out, bar
