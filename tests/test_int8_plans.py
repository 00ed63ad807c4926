"""The rules on sizes of the products in 8-bit integers (no GPU): what the launches and workspaces that follow from them rely on."""
import random

import pytest

from tests import int8_plans

SIZES = [(1, 16), (1, 1 << 30), (16, 28672), (77, 4096), (8192, 28672), (0x7FFFFF00, 8), (0x7FFFFF00, 0x7FFFFF00), (3, 0x7FFFFF00), (100000, 100000)]


def drawn(n=400):
    r = random.Random(4)
    return [(int(2 ** r.uniform(0, 14)), int(2 ** r.uniform(0, 16)), 16 * int(2 ** r.uniform(0, 13)), r.choice([0, 0, 1, 4, 8, 64, 1024])) for _ in range(n)]


@pytest.mark.parametrize("K", [16, 4096, 131072])
@pytest.mark.parametrize("E", [0, 1, 64, 1024])
def test_launches_fit(K, E):
    """Less than 2^32 threads, 256 to a workgroup, where tiles are not looped over."""
    for T, N in SIZES:
        f = int8_plans.form(T, N, K, E)
        assert f.looped or f.grid <= int8_plans.most_workgroups() < 1 << 24, (T, N, f)


def test_partial_sums_fit():
    for T, N, K, E in drawn():
        f = int8_plans.form(T, N, K, E)
        assert f.part <= int8_plans.part_limit()
        assert f.ranges == 1 or (E == 0 and f.name in ("mid32", "mid64", "mid96", "deep128") and -(-K // 128) >= 2 * f.ranges)
        # the form of a workspace that was sized for the call, and of one that has no room
        assert int8_plans.form(T, N, K, E, f.part)[:2] == f[:2]
        assert int8_plans.form(T, N, K, E, 0).ranges == 1
        if f.part:
            assert int8_plans.form(T, N, K, E, f.part - 1).part < f.part


def test_single_tokens_fit():
    for T, N, K, E in drawn(2000):
        f = int8_plans.form(T, N, K, E)
        if f.single:
            # eight tokens' sums, at most; codes in LDS beside the partial sums; 64 values to each of 256 threads
            assert T <= 8 and T * (K + 16) <= 131072 and K <= 16384
    assert int8_plans.form(1, 4096, 4096).single == 1 and int8_plans.form(1, 28672, 4096).single == 2
    assert not int8_plans.form(4, 4096, 4096).single and int8_plans.form(4, 4096, 4096, 8).single
    assert not int8_plans.form(1, 4096, 16400).single and int8_plans.form(5, 4096, 4096, 8).single and int8_plans.form(8, 4096, 4096, 8).single
    assert not int8_plans.form(9, 1024, 1024, 64).single and not int8_plans.form(8, 4096, 14336, 8).single and not int8_plans.form(8, 18432, 2304, 8).single
