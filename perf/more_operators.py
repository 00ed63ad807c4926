"""What decoding with group scales and layers of experts is measured on.

A server keeps a model's weights as r-bit codes with one scale and one zero-point for every `group` inputs of a row, packed as
this library packs planes, and decodes up to 16 sequences at a time.  Its feed-forward blocks may be split over experts; a
router's scores choose some of them for each token, and in training the router learns from the gradient of its weights.  Four
kinds of passes:

    gemv        the matrix-vector products of up to 16 tokens with a plane that has group scales
    choose      a router's scores to the experts of each token and their weights
    choose_bwd  the gradient of the weights back to the scores
    layer       a whole feed-forward layer of experts for up to 16 tokens: gated products, down products, weighted sum

Sizes are those of `synth.py`, the tests and `bench.py` (2304 x 9216, 4096 x 14336, 4608 x 36864) and generic ones, groups of 32
to 128 inputs, generic expert counts.
"""
from __future__ import annotations

import math
import zlib

import torch

own = False


def listed():
    return [
        # -- matrix-vector products -------------------------------------------------------------------------------------
        # one sequence through a square 7B-shaped projection: the smallest product, latency
        {"name": "gemv_one", "kind": "gemv", "B": 1, "N": 4096, "K": 4096, "group": 128, "r": 4},
        # three sequences at two bits, short groups, a number of rows that is no multiple of anything
        {"name": "gemv_two_bits", "kind": "gemv", "B": 3, "N": 9217, "K": 2304, "group": 64, "r": 2},
        # a full decode batch through the long rows of a down projection, groups of 32
        {"name": "gemv_batch", "kind": "gemv", "B": 16, "N": 4096, "K": 14336, "group": 32, "r": 4},
        # one sequence through a stacked gate / up plane of the 27B-shaped model: the largest product, bandwidth
        {"name": "gemv_tall", "kind": "gemv", "B": 1, "N": 73728, "K": 4608, "group": 128, "r": 4},
        # -- the router's choice ----------------------------------------------------------------------------------------
        # a decode step of 16 sequences, many experts: latency
        {"name": "choose_step", "kind": "choose", "M": 16, "E": 64, "top": 8, "renormalize": False, "masked": 0.0},
        # a long training batch, some tokens padding and some experts not to be had
        {"name": "choose_long", "kind": "choose", "M": 65531, "E": 128, "top": 8, "renormalize": True, "masked": 0.1},
        # the gradient of a small training batch, weights normalized over the chosen
        {"name": "choose_bwd_short", "kind": "choose_bwd", "M": 509, "E": 8, "top": 2, "renormalize": True, "masked": 0.0},
        # the gradient of a long one, weights as the softmax over all experts gives them
        {"name": "choose_bwd_long", "kind": "choose_bwd", "M": 65531, "E": 64, "top": 6, "renormalize": False, "masked": 0.1},
        # -- whole layers -------------------------------------------------------------------------------------------------
        # one token, eight of many small experts
        {"name": "layer_one", "kind": "layer", "B": 1, "top": 8, "E": 64, "d": 2048, "F": 1024, "group": 128, "r": 4, "gate": "silu", "masked": 0.0},
        # five tokens of a 2B-shaped layer at two bits
        {"name": "layer_two_bits", "kind": "layer", "B": 5, "top": 2, "E": 8, "d": 2304, "F": 9216, "group": 64, "r": 2, "gate": "gelu", "masked": 0.0},
        # a decode batch over many small experts, some of its places empty
        {"name": "layer_batch", "kind": "layer", "B": 16, "top": 4, "E": 128, "d": 2048, "F": 1408, "group": 128, "r": 4, "gate": "silu", "masked": 0.2},
        # a full decode batch of a 7B-shaped layer, nearly every expert chosen: the largest
        {"name": "layer_full", "kind": "layer", "B": 16, "top": 2, "E": 8, "d": 4096, "F": 14336, "group": 128, "r": 4, "gate": "silu", "masked": 0.0},
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in lo..hi, spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(-(-lo // step), min(hi // step, round(v / step))) * step


def draw(rng):
    kind = rng.choice(["gemv", "gemv", "gemv", "choose", "choose_bwd", "layer", "layer", "layer"])
    r, group = rng.choice([4, 4, 4, 4, 2, 8]), rng.choice([32, 64, 128, 128, 256])
    group = max(group, 128 // r)  # 16 bytes of codes at least
    while True:
        if kind == "gemv":
            c = {"kind": kind, "B": rng.choice([1, 1, 2, 4, 16, rng.randint(1, 16)]), "N": _log(rng, 256, 73728), "K": _log(rng, 1024, 16384, group),
                 "group": group, "r": r}
            if c["N"] * c["K"] * r <= 73728 * 4608 * 4:
                return c
        elif kind == "layer":
            c = {"kind": kind, "B": rng.choice([1, 1, 2, 4, 16, rng.randint(1, 16)]), "top": rng.randint(1, 8), "E": rng.choice([8, 16, 60, 64, 128])}
            c.update(d=_log(rng, 512, 4096, group), F=_log(rng, 512, 14336, group), group=group, r=r, gate=rng.choice(["silu", "gelu"]),
                     masked=rng.choice([0.0, 0.0, 0.2]))
            if c["E"] * c["d"] * c["F"] * r <= 8 * 4096 * 14336 * 4:
                return c
        else:
            E = rng.choice([4, 8, 16, 32, 60, 64, 128, 256, rng.randint(2, 300)])
            c = {"kind": kind, "M": _log(rng, 1, 65536), "E": E, "top": rng.randint(1, min(8, E)), "renormalize": rng.random() < 0.5,
                 "masked": rng.choice([0.0, 0.1])}
            return c


# --------------------------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------------------------
class _Rand:
    """Seeded draws on the GPU."""

    def __init__(self, seed, what):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed((seed * 1_000_003 + zlib.crc32(what.encode())) % (1 << 62))

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda")

    def tokens(self, M, K):
        """bf16 N(0, 1) times a size for each token, one feature of a hundred eight times as large."""
        x = self.normal(M, K) * torch.exp(0.5 * self.normal(M, 1))
        x *= torch.where(self.uniform(K) < 0.01, 8.0, 1.0)
        return x.to(torch.bfloat16)

    def plane(self, rows, K, group, r):
        """Normal weights that keep outputs at about the inputs' size: 8-bit codes over the range of each group, sliced to r bits
        (rounded up at the halves, the top code clamped), packed along K from the low bits up; scale and zero-point of each group."""
        packed = torch.empty(rows, K * r // 8, dtype=torch.uint8, device="cuda")
        alpha = torch.empty(rows, K // group, dtype=torch.bfloat16, device="cuda")
        zero = torch.empty_like(alpha)
        per = max(1, (1 << 26) // K)
        for at in range(0, rows, per):
            n = min(per, rows - at)
            w = self.normal(n, K // group, group) / math.sqrt(K)
            lo, hi = w.amin(2, keepdim=True), w.amax(2, keepdim=True)
            a = (hi - lo) / 255.0
            z = -lo / a
            q = (w / a + z).round_().clamp_(0, 255).to(torch.uint8).view(n, K)
            if r < 8:
                q = torch.clamp((q.to(torch.int16) + (1 << (7 - r))) >> (8 - r), max=(1 << r) - 1).to(torch.uint8)
            q = q.view(n, K * r // 8, 8 // r)
            out = q[:, :, 0].clone()
            for j in range(1, 8 // r):
                out |= q[:, :, j] << (r * j)
            packed[at:at + n], alpha[at:at + n], zero[at:at + n] = out, a[:, :, 0], z[:, :, 0]
        return packed, alpha, zero

    def scores(self, M, E, masked):
        """A router's scores (experts of unequal popularity); with `masked` that share of tokens has no expert at all (padding) and half
        that share of the pairs is not to be had."""
        s = 1.5 * self.normal(M, E) + 0.5 * self.normal(1, E)
        if masked:
            s[self.uniform(M, E) < masked / 2] = -math.inf
            s[self.uniform(M) < masked] = -math.inf
        return s


def prepare(case, seed):
    c = case
    rnd = _Rand(seed, c["kind"])
    s = {"case": c, "kept": {}}
    if c["kind"] == "gemv":
        s["x"] = rnd.tokens(c["B"], c["K"])
        s["packed"], s["alpha"], s["zero"] = rnd.plane(c["N"], c["K"], c["group"], c["r"])
        return s
    if c["kind"] == "layer":
        B, top, E, d, F = c["B"], min(c["top"], c["E"]), c["E"], c["d"], c["F"]
        s["x"] = rnd.tokens(B, d)
        best, ids = rnd.scores(B, E, 0.0).topk(top, dim=1)
        ids = ids.to(torch.int32)
        if c["masked"]:
            ids[rnd.uniform(B) < c["masked"]] = -1
        s["ids"], s["weight"] = ids.contiguous(), torch.softmax(best, dim=1).contiguous()
        L = {"r": c["r"]}
        for name, rows, K in (("gate_up", 2 * F, d), ("down", d, F)):
            packed, alpha, zero = rnd.plane(E * rows, K, c["group"], c["r"])
            short = "gu" if name == "gate_up" else "dn"
            L.update({name: packed.view(E, rows, -1), "alpha_" + short: alpha.view(E, rows, -1), "zero_" + short: zero.view(E, rows, -1)})
        s["layer"] = L
        return s
    s["scores"] = rnd.scores(c["M"], c["E"], c["masked"])
    if c["kind"] == "choose_bwd":
        s["ids"], s["weight"] = _plain_choose(s, c).values()  # what the forward left
        s["dweight"] = rnd.normal(c["M"], c["top"]) / c["M"]
    return s


# --------------------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state, state["case"])


def _kept(s, name, make):
    """A buffer that the program keeps from pass to pass."""
    if name not in s["kept"]:
        s["kept"][name] = make()
    return s["kept"][name]


def _empty(s, name, *shape, dtype=torch.bfloat16):
    return _kept(s, name, lambda: torch.empty(*shape, dtype=dtype, device="cuda"))


def _own_gemv(s, c):
    import paper_2502_06786_amd as mq
    return mq.mq_gemv_grouped(s["x"], s["packed"], s["alpha"], s["zero"], c["r"], c["K"], c["group"], y=_empty(s, "y", c["B"], c["N"]))


def _own_choose(s, c):
    import paper_2502_06786_amd as mq
    ids, weight = mq.mq_experts_choose(s["scores"], c["top"], renormalize=c["renormalize"],
                                       ids=_empty(s, "ids", c["M"], c["top"], dtype=torch.int32),
                                       weight=_empty(s, "weight", c["M"], c["top"], dtype=torch.float32))
    return {"ids": ids, "weight": weight}


def _own_choose_bwd(s, c):
    import paper_2502_06786_amd as mq
    return mq.mq_experts_choose_bwd(s["scores"], s["ids"], s["weight"], s["dweight"], renormalize=c["renormalize"],
                                    dscores=_empty(s, "dscores", c["M"], c["E"], dtype=torch.float32))


def _own_layer(s, c):
    import paper_2502_06786_amd as mq
    ws = _kept(s, "ws", lambda: torch.empty(max(16, mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_FFN, s["ids"].numel(), c["F"], c["d"], 1)),
                                            dtype=torch.uint8, device="cuda"))
    return mq.mq_experts_ffn(s["x"], s["layer"], s["ids"], s["weight"], c["F"], c["group"], silu=c["gate"] == "silu",
                             y=_empty(s, "y", c["B"], c["d"]), ws=ws)


_OWN = {"gemv": _own_gemv, "choose": _own_choose, "choose_bwd": _own_choose_bwd, "layer": _own_layer}


def _weights(packed, alpha, zero, r):
    """alpha (2^(8-r) code - zero) of every weight, [rows, K] in 32 bits."""
    shift = torch.arange(0, 8, r, device=packed.device, dtype=torch.uint8)
    codes = ((packed.unsqueeze(-1) >> shift) & ((1 << r) - 1)).float() * float(1 << (8 - r))
    codes = codes.view(*alpha.shape, -1)  # [..., rows, groups, group]
    w = (codes - zero.float().unsqueeze(-1)) * alpha.float().unsqueeze(-1)
    return w.flatten(-2)


def _plain_gemv(s, c):
    return (s["x"].float() @ _weights(s["packed"], s["alpha"], s["zero"], c["r"]).t()).to(torch.bfloat16)


def _plain_choose(s, c):
    scores = s["scores"]
    best, ids = torch.sort(scores, dim=1, descending=True, stable=True)  # equal scores: the lowest index first
    best, ids = best[:, :c["top"]], ids[:, :c["top"]]
    live = best > -math.inf
    most = torch.where(live[:, :1], best[:, :1], 0.0)
    e = torch.exp(best - most)
    total = (e if c["renormalize"] else torch.exp(scores - most)).sum(1, keepdim=True)
    return {"ids": torch.where(live, ids, -1).to(torch.int32), "weight": torch.where(live, e / torch.where(total > 0, total, 1.0), 0.0)}


def _plain_choose_bwd(s, c):
    ids, live = s["ids"].long().clamp(min=0), s["ids"] >= 0
    dw = torch.where(live, s["dweight"], 0.0)
    mean = (dw * s["weight"]).sum(1, keepdim=True)
    if c["renormalize"]:
        return torch.zeros_like(s["scores"]).scatter_add_(1, ids, s["weight"] * torch.where(live, dw - mean, 0.0))
    most = s["scores"].amax(1, keepdim=True)
    e = torch.exp(s["scores"] - torch.where(most > -math.inf, most, 0.0))
    total = e.sum(1, keepdim=True)
    p = e / torch.where(total > 0, total, 1.0)
    return p * (torch.zeros_like(p).scatter_add_(1, ids, dw) - mean)


def _act(g, gate):
    if gate == "silu":
        return g / (1.0 + torch.exp(-g))
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))


def _plain_layer(s, c):
    """Every choice with its own copy of its expert's weights, or, where there are more choices than experts, every expert with all tokens."""
    L, ids, x = s["layer"], s["ids"].long(), s["x"].float()
    B, top = ids.shape
    weight = torch.where(ids >= 0, s["weight"], 0.0)
    if B * top < c["E"]:
        e = ids.clamp(min=0).reshape(-1)
        of = (torch.arange(B * top, device="cuda") // top == torch.arange(B, device="cuda")[:, None]) * weight.reshape(-1)  # [B, choices]
    else:
        e = torch.arange(c["E"], device="cuda")
        of = ((ids[:, :, None] == e) * weight[:, :, None]).sum(1)
    n = e.numel()
    w = _weights(L["gate_up"][e], L["alpha_gu"][e], L["zero_gu"][e], c["r"])
    g, u = (w.view(n * 2 * c["F"], c["d"]) @ x.t()).view(n, c["F"], 2, B).unbind(2)
    a = _act(g, c["gate"]) * u  # [n, F, B]
    o = torch.bmm(_weights(L["down"][e], L["alpha_dn"][e], L["zero_dn"][e], c["r"]), a)  # [n, d, B]
    return (o.permute(2, 0, 1) * of[:, :, None]).sum(1).to(torch.bfloat16)


_PLAIN = {"gemv": _plain_gemv, "choose": _plain_choose, "choose_bwd": _plain_choose_bwd, "layer": _plain_layer}


# --------------------------------------------------------------------------------------------------------------------
# floors
# --------------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "gemv":
        B, N, K = c["B"], c["N"], c["K"]
        return {"bytes": N * (K * c["r"] // 8 + 4 * (K // c["group"])) + 2 * B * (N + K), "flops": 2 * B * N * K}
    if c["kind"] == "layer":
        B, top, E, d, F = c["B"], min(c["top"], c["E"]), c["E"], c["d"], c["F"]
        used = E * (1.0 - (1.0 - top / E) ** (B * (1.0 - c["masked"])))  # experts that some token chooses, were all equally popular
        return {"bytes": used * 3 * d * F * (c["r"] / 8 + 4 / c["group"]) + 4 * B * d + 8 * B * top, "flops": 6 * B * (1.0 - c["masked"]) * top * d * F}
    M, E, top = c["M"], c["E"], c["top"]
    if c["kind"] == "choose":
        return {"bytes": M * (4 * E + 8 * top), "flops": M * (4 * E + E * top)}
    return {"bytes": M * ((4 if c["renormalize"] else 8) * E + 12 * top), "flops": M * (6 * E + 4 * top)}


# --------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------------------------------------------------
def _exact_product(x, packed, alpha, zero, r):
    """x [B, K] times the rows of a plane, a bit position of the packed bytes at a time: [B, rows]."""
    B, K = x.shape
    rows, groups = alpha.shape
    per = 8 // r
    xs = x.double().view(B, groups, K // groups // per, per)
    a, z = alpha.double(), zero.double()
    y = -(xs.sum((2, 3)) @ (a * z).t())
    for at in range(0, rows, max(1, (1 << 27) // K)):
        part = slice(at, min(rows, at + max(1, (1 << 27) // K)))
        b = packed[part].view(-1, groups, K // groups // per).to(torch.int32)
        for j in range(per):
            code = (torch.div(b, 1 << (r * j), rounding_mode="floor") % (1 << r)).double() * (a[part] * 2.0 ** (8 - r))[..., None]
            y[:, part] += xs[..., j].reshape(B, -1) @ code.view(code.shape[0], -1).t()
    return y


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "gemv":
        return _exact_product(s["x"], s["packed"], s["alpha"], s["zero"], c["r"])
    if c["kind"] == "layer":
        L = s["layer"]
        out = torch.zeros(c["B"], c["d"], dtype=torch.float64, device="cuda")
        for e in range(c["E"]):
            token, choice = (s["ids"] == e).nonzero(as_tuple=True)
            if not token.numel():
                continue
            h = _exact_product(s["x"][token], L["gate_up"][e], L["alpha_gu"][e], L["zero_gu"][e], c["r"])
            g, u = h[:, 0::2], h[:, 1::2]
            t = g if c["gate"] == "silu" else 2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)
            o = _exact_product(g * torch.sigmoid(t) * u, L["down"][e], L["alpha_dn"][e], L["zero_dn"][e], c["r"])
            out.index_add_(0, token, o * s["weight"][token, choice].double()[:, None])
        return out
    scores = s["scores"].double()
    whole = torch.softmax(scores, dim=1).nan_to_num(0.0)  # rows without any expert
    if c["kind"] == "choose":
        w = whole.sort(dim=1, descending=True).values[:, :c["top"]]
        if c["renormalize"]:
            w = (w / w.sum(1, keepdim=True)).nan_to_num(0.0)
        return {"ids": None, "weight": w}
    # the derivative of sum(dweight * weight) by the scores, the choices held
    live = s["ids"] >= 0
    at = torch.where(live, s["ids"].long(), c["E"])
    x = torch.cat([scores, scores.new_full((c["M"], 1), -math.inf)], 1).gather(1, at) if c["renormalize"] else scores
    p = torch.softmax(x, dim=1).nan_to_num(0.0)
    up = torch.where(live, s["dweight"].double(), 0.0)
    if not c["renormalize"]:
        up = torch.zeros(c["M"], c["E"] + 1, dtype=torch.float64, device="cuda").scatter_add_(1, at, up)[:, :c["E"]]
    dx = p * up - p * (p * up).sum(1, keepdim=True)
    if not c["renormalize"]:
        return dx
    return torch.zeros(c["M"], c["E"] + 1, dtype=torch.float64, device="cuda").scatter_add_(1, at, dx)[:, :c["E"]]
