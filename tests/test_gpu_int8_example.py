"""examples/int8_experts.py at small sizes."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "int8_experts.py")


@pytest.mark.parametrize("args", [["--tokens", "37"], ["--tokens", "3", "--bits", "4", "--gate", "silu", "--experts", "3", "--top", "1"]])
def test_example(args):
    spec = importlib.util.spec_from_file_location("int8_experts", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    lines = module.main(args + ["--d", "256", "--f", "512"])   # (tokens alone are compared with the prompt's inside, bit by bit)
    assert [line["what"] for line in lines] == ["feed-forward block", "layer of experts"]
    # Two quantizations of normal values to steps of top / 127 with top about 3 to 4 deviations: an error of 4 / 127 / sqrt(12) = 0.9 % of a
    # deviation each, twice through a product that adds independent errors; the gate's output is heavier-tailed (top up to 10 deviations).
    assert all(0 < line["off"] < 0.04 for line in lines), lines
