"""Which places and channels the workgroups of the products in 8-bit integers take (csrc/mq_int8_blocks.h), on the host: bounds of experts as
the grouping writes them, and bounds that hold anything, which the header promises to keep inside the arrays."""
import os
import subprocess

from tests.plans import CSRC

SOURCE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "int8_blocks.cpp")


def test_blocks(tmp_path):
    program = str(tmp_path / "blocks")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unknown-pragmas", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, SOURCE, "-o", program], check=True)
    run = subprocess.run([program], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.startswith("ok "), (run.stdout[-2000:], run.stderr[-2000:])
