"""The rules on sizes of the products in 8-bit integers (csrc/mq_int8_plan.h) for tests that have to know which form a call takes: built with
the host compiler on first use, no GPU needed."""
import ctypes
import functools
import os
import subprocess
import tempfile
from collections import namedtuple

from tests.plans import CSRC

SOURCE = r'''
#include "mq_int8_plan.h"
using namespace mq;
extern "C" void int8_form(int64_t T, int64_t N, int64_t K, int64_t E, int64_t part_bytes, int64_t *out) {
    const Int8Plan p = make_int8_plan(T, N, K, E, part_bytes);
    const Int8Cost &f = kInt8Costs[p.form];
    out[0] = p.form, out[1] = p.splits, out[2] = int8_grid(p.form, T, N, E, p.splits), out[3] = f.looped;
    out[4] = E == 0 ? int8_part_bytes(f, T, N, p.splits) : 0;
    out[5] = f.places == 256 && int8_quarters(out[2]);
    out[6] = int8_single(T, N, K, E) ? 1 + int8_single_wide(T, N, E) : 0;
}
extern "C" int64_t int8_part_limit(void) { return kInt8PartBytes; }
extern "C" int64_t int8_most_workgroups(void) { return kInt8MostWorkgroups; }
'''

FORMS = ["few", "mid32", "mid64", "mid96", "deep128", "tile128", "tile256"]
# grid: workgroups, or tiles where they are looped over (`looped`); part: bytes of partial sums; quarters: the last round of 256-tiles is
# done in 128-tiles (dense products); single: 0, or 1 / 2 where bf16 tokens are quantized by workgroups of 16 / 32 channels
Form = namedtuple("Form", "name ranges grid looped part quarters single")


@functools.lru_cache(maxsize=None)
def _lib():
    folder = tempfile.mkdtemp(prefix="int8_plans_")
    src, lib = os.path.join(folder, "plans.cpp"), os.path.join(folder, "plans.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", CSRC, src, "-o", lib], check=True)
    out = ctypes.CDLL(lib)
    i64 = ctypes.c_int64
    out.int8_form.argtypes = [i64, i64, i64, i64, i64, ctypes.POINTER(i64)]
    out.int8_part_limit.restype = out.int8_most_workgroups.restype = i64
    return out


def form(T, N, K, E=0, part_bytes=None):
    """E = 0: a dense product."""
    out = (ctypes.c_int64 * 7)()
    _lib().int8_form(T, N, K, E, part_limit() if part_bytes is None else part_bytes, out)
    return Form(FORMS[out[0]], out[1], out[2], bool(out[3]), out[4], bool(out[5]), out[6])


def part_limit():
    return _lib().int8_part_limit()


def most_workgroups():
    return _lib().int8_most_workgroups()
