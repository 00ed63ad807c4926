"""A feed-forward block and a layer of experts served in 8-bit integers.

Weights are quantized once (one int8 code each) and read at r bits; then a prompt goes through in one call of each kind, and its last
tokens one at a time, as a server decodes.  Both give the same bits: sums of whole numbers have no order.  The results are compared with
the same sliced weights on bf16 tokens in fp32, which says what the tokens' own 8 bits cost.

    python examples/int8_experts.py [--tokens 512] [--experts 8] [--top 2] [--d 2304] [--f 9216] [--bits 8] [--gate gelu]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2502_06786_amd as mq  # noqa: E402


class Weights:
    """E layers, W fp32 [E, N, K], as codes of r bits, a byte each, with their scale and zero-point for each channel."""

    def __init__(self, W, r):
        E, N, K = W.shape
        Q, alpha, zero = mq.mq_quantize_int8(W.view(E * N, K))
        self.codes = (Q if r == 8 else mq.mq_slice(Q, r)).view(E, N, K)
        self.alpha, self.zero, self.r = alpha.view(E, N), zero.view(E, N), r

    def floats(self, e):
        """alpha (2^(8-r) code - zero)"""
        return self.alpha[e, :, None] * (self.codes[e].float() * 2.0 ** (8 - self.r) - self.zero[e, :, None])


class Buffers:
    """What calls on up to `tokens` tokens write, allocated once."""

    def __init__(self, tokens, top, E, d, F):
        T = tokens * top
        new = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.offsets, self.rows, self.place = new(E + 1, dtype=torch.int32), new(T, dtype=torch.int32), new(tokens, top, dtype=torch.int32)
        self.hidden, self.each, self.out = new(T, F), new(T, d), new(tokens, d)
        sizes = [mq.mq_workspace_bytes(mq.MQ_OP_EXPERTS_ROUTE, T, E, 0, 1)]
        for op in (mq.MQ_OP_LINEAR_FWD_INT8, mq.MQ_OP_EXPERTS_FWD_INT8):
            sizes += [mq.mq_workspace_bytes(op, T, 2 * F, d, 1), mq.mq_workspace_bytes(op, T, d, F, 1)]
        self.ws = new(max(sizes), dtype=torch.uint8)


def feed_forward(x, up, down, gate, b):
    """down(act(gate) * up), the gate in the first product's epilogue: x bf16 [M, d] -> [M, d]"""
    M = len(x)
    h = mq.mq_linear_fwd_int8(x, up.codes[0], up.alpha[0], up.zero[0], up.r, gate=gate, Y=b.hidden[:M], ws=b.ws)
    return mq.mq_linear_fwd_int8(h, down.codes[0], down.alpha[0], down.zero[0], down.r, Y=b.out[:M], ws=b.ws)


def experts(x, ids, weight, up, down, gate, b):
    """sum over j of weight[m, j] expert ids[m, j] (x[m])"""
    M, top = ids.shape
    T, E = M * top, len(up.codes)
    offsets, rows, place = mq.mq_experts_route(ids, E, b.offsets, b.rows[:T], b.place[:M], ws=b.ws)
    h = mq.mq_experts_fwd_int8(x, offsets, up.codes, up.alpha, up.zero, up.r, rows=rows, gate=gate, Y=b.hidden[:T], ws=b.ws)
    y = mq.mq_experts_fwd_int8(h, offsets, down.codes, down.alpha, down.zero, down.r, Y=b.each[:T], ws=b.ws)
    return mq.mq_experts_combine(y, place, weight, b.out[:M])


def plain(x, e, up, down, gate):
    """one expert with the same weights on unquantized tokens, in fp32"""
    g, u = (x.float() @ up.floats(e).t()).view(len(x), -1, 2).unbind(2)
    act = torch.nn.functional.silu(g) if gate == "silu" else torch.nn.functional.gelu(g, approximate="tanh")
    return (act * u) @ down.floats(e).t()


def microseconds(f, n=50):
    f()
    first, last = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    first.record()
    for _ in range(n):
        f()
    last.record()
    last.synchronize()
    return first.elapsed_time(last) / n * 1e3


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--tokens", type=int, default=512)
    p.add_argument("--experts", type=int, default=8)
    p.add_argument("--top", type=int, default=2)
    p.add_argument("--d", type=int, default=2304)
    p.add_argument("--f", type=int, default=9216)
    p.add_argument("--bits", type=int, default=8)
    p.add_argument("--gate", choices=["gelu", "silu"], default="gelu")
    a = p.parse_args(argv)
    M, E, d, F = a.tokens, a.experts, a.d, a.f

    g = torch.Generator(device="cuda").manual_seed(0)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    up = Weights(randn(E, 2 * F, d) * d ** -0.5, a.bits)   # channels 2f, 2f + 1: gate and up of feature f
    down = Weights(randn(E, d, F) * F ** -0.5, a.bits)
    x = randn(M, d).to(torch.bfloat16)
    chance = torch.softmax(x.float() @ (randn(d, E) * d ** -0.5), 1)
    weight, ids = chance.topk(a.top, dim=1)
    weight, ids = (weight / weight.sum(1, keepdim=True)).contiguous(), ids.to(torch.int32).contiguous()
    b, one = Buffers(M, a.top, E, d, F), Buffers(1, a.top, E, d, F)

    lines = []
    for name, call, want in (
            ("feed-forward block", lambda x, ids, w, b: feed_forward(x, up, down, a.gate, b), lambda: plain(x, 0, up, down, a.gate)),
            ("layer of experts", lambda x, ids, w, b: experts(x, ids, w, up, down, a.gate, b),
             lambda: sum(torch.where(ids == e, weight, 0.0).sum(1, keepdim=True) * plain(x, e, up, down, a.gate) for e in range(E)))):
        prompt = call(x, ids, weight, b).clone()
        for m in range(max(0, M - 4), M):
            single = call(*(t[m:m + 1].clone() for t in (x, ids, weight)), one)   # (pointers are 16-byte aligned: no views)
            assert torch.equal(single[0].view(torch.int16), prompt[m].view(torch.int16)), "a token alone differs from the same one in the prompt"
        want = want()
        off = float((prompt.double() - want.double()).norm() / want.double().norm())
        x1, ids1, w1 = (t[:1].clone() for t in (x, ids, weight))
        t, t1 = microseconds(lambda: call(x, ids, weight, b)), microseconds(lambda: call(x1, ids1, w1, one))
        lines.append({"what": name, "tokens": M, "us": t, "us_single": t1, "off": off})
        print(f"{name}: {M} tokens {t:.1f} us, one token {t1:.1f} us; the tokens' 8 bits change the result by {100 * off:.2f} %", flush=True)
    return lines


if __name__ == "__main__":
    main()
