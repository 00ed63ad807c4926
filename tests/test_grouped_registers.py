"""Registers of the compiled kernels of products with group scales (csrc/mq_grouped.h): none keeps registers in memory.  Its reloads would wait, in
order, for every piece that is under way."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2502_06786_amd import build as mq_build
from tests.test_registers import OBJDUMP, READELF


def test_no_registers_in_memory(tmp_path):
    if not os.path.exists(mq_build.LIB):
        pytest.fail(f"{mq_build.LIB} is not built (python -c 'import __graft_entry__ as g; g.build()')")
    if not (os.path.exists(OBJDUMP) and os.path.exists(READELF)):
        pytest.skip("no llvm-objdump and llvm-readelf")
    shutil.copy(mq_build.LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    seen = {}
    for name in os.listdir(tmp_path):
        if "gfx950" in name:
            notes = subprocess.run([READELF, "--notes", name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
            for kernel in notes.split(".agpr_count")[1:]:
                m = re.search(r"\.name:\s+_ZN2mq\d+(gemv_grouped|experts_gate_up|experts_down|choose|choose_bwd)_kernel", kernel)
                if m:
                    seen.setdefault(m.group(1), []).append(int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", kernel).group(1)))
    assert sorted(seen) == ["choose", "choose_bwd", "experts_down", "experts_gate_up", "gemv_grouped"]
    assert not any(any(sizes) for sizes in seen.values()), seen
