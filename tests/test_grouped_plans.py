"""The sizes at which the products with group scales are compared with their definition reach every form that they can take (no GPU)."""
import numpy as np
import torch

from tests import grouped_plans as plans, grouped_reference as ref


def test_sizes_reach_every_product():
    seen = set()
    for r, group, B, N, K in plans.products():
        assert K % group == 0 and N % 16 != 0
        f = plans.rules(r, group, B=B, N=N)
        assert K % f.stretch != 0
        seen.add((r, f.chunk, f.tokens, f.gemv))
    assert seen == {(r, c, t, tiles) for r, c in plans.CHUNKS for t in (4, 8, 16) for tiles in (1, 2)} - {(4, 32, 4, 2)}


def test_sizes_reach_every_layer():
    gate_up, down, both = set(), set(), set()
    for r, group, B, top, E, d, F in plans.layers():
        assert d % group == 0 and F % group == 0
        f = plans.rules(r, group, B=B, d=d, F=F, experts=min(B * top, E))
        gate_up.add((r, f.chunk, f.tokens, f.gate_up))
        down.add((r, f.chunk, 4 if B <= 4 else 8, f.down, f.splits > 1))
        both.add((r, f.gate_up, f.down))
    assert gate_up == {(r, c, t, tiles) for r, c in plans.CHUNKS for t in (4, 8, 16) for tiles in (1, 2)}
    assert {f[:4] for f in down} == {(r, c, t, tiles) for r, c in plans.CHUNKS for t in (4, 8) for tiles in (1, 2)}
    assert {f[0:1] + f[3:] for f in down} == {(r, tiles, shared) for r in (2, 4, 8) for tiles in (1, 2) for shared in (False, True)}
    assert both == {(r, a, b) for r in (2, 4, 8) for a in (1, 2) for b in (1, 2)}


def test_definitions_on_tensors():
    """The definitions on tensors, which the large sizes are compared with, are those on arrays."""
    rng = np.random.default_rng(1)
    for r in (8, 4, 2):
        E, d, F, group, B = 3, 128, 192, 64, 4
        host, dev = {}, {}
        for short, rows, K in (("gu", 2 * F, d), ("dn", d, F)):
            host["codes_" + short] = rng.integers(0, 1 << r, (E, rows, K))
            host["alpha_" + short], host["zero_" + short] = 0.01 * rng.random((E, rows, K // group)), 200 * rng.random((E, rows, K // group))
            dev["packed_" + short] = torch.from_numpy(ref.pack(host["codes_" + short], r))
            dev["alpha_" + short], dev["zero_" + short] = torch.from_numpy(host["alpha_" + short]), torch.from_numpy(host["zero_" + short])
        x, weight = rng.standard_normal((B, d)), rng.random((B, 2))
        ids = rng.integers(-1, E + 1, (B, 2))
        y, bar = ref.product(x, host["codes_gu"][1], host["alpha_gu"][1], host["zero_gu"][1], r)
        got, far = ref.product_on(torch.from_numpy(x), dev["packed_gu"][1], dev["alpha_gu"][1], dev["zero_gu"][1], r)
        assert np.allclose(got.numpy(), y, rtol=1e-10, atol=1e-10) and np.allclose(far.numpy(), bar, rtol=1e-10)
        for silu, residual in ((True, False), (False, True)):
            y, bar = ref.layer(x, host, ids, weight, r, silu, residual)
            got, far = ref.layer_on(torch.from_numpy(x), dev, torch.from_numpy(ids), torch.from_numpy(weight), r, silu, residual)
            assert np.allclose(got.numpy(), y, rtol=1e-10, atol=1e-8) and np.allclose(far.numpy(), bar, rtol=1e-10, atol=1e-12)
