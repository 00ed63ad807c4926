"""The waits around the 8-bit matrix products that are written as inline assembly (csrc/mq_int8_tile.hip), in the compiled library: the rules
and the scan of tests/test_matrix_waits.py, which the 16x16x64 product shares with the 16x16x32 one (both occupy the matrix core for sixteen
cycles)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2502_06786_amd import build as mq_build
from tests.test_matrix_waits import OBJDUMP, parse, violations

KERNELS = re.compile(r"_ZN2mq\d+int8_tile_kernelI")


def test_products_of_the_tiles(tmp_path):
    if not os.path.exists(mq_build.LIB):
        pytest.fail(f"{mq_build.LIB} is not built (python -c 'import __graft_entry__ as g; g.build()')")
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    shutil.copy(mq_build.LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    kernels = products = loads = 0
    for name in sorted(os.listdir(tmp_path)):
        if "gfx950" not in name:
            continue
        text = subprocess.run([OBJDUMP, "-d", name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]{16} <)", text):
            m = re.match(r"[0-9a-f]{16} <([^>]+)>:", part)
            if not m or not KERNELS.match(m.group(1)):
                continue
            code = parse(part.split("\n")[1:])
            kernels += 1
            products += sum(c[4] for c in code)
            loads += sum(c[0].endswith(" lds") for c in code)
            assert not violations(code), (m.group(1), violations(code)[:3])
    assert kernels == 8 and products > 300 and loads > 100
