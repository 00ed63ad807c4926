"""The rules on sizes of the products with group scales (csrc/mq_grouped_plan.h) for tests that have to know which form a call takes: built with
the host compiler on first use, no GPU needed."""
import ctypes
import functools
import os
import subprocess
import tempfile
from collections import namedtuple

from tests.plans import CSRC

SOURCE = r'''
#include "mq_grouped_plan.h"
using namespace mq;
extern "C" void grouped_rules(int r, int64_t group, int64_t B, int64_t N, int64_t d, int64_t F, int64_t experts, int64_t *out) {
    const int c = chunk_codes(r, group);
    out[0] = c, out[1] = stretch_codes(r), out[2] = token_class(B), out[3] = gemv_tiles(r, c, B, N), out[4] = gate_up_tiles(F, experts);
    out[5] = down_tiles(r, d, F, experts), out[6] = down_splits(r, d, F, experts, (int)out[5]);
}
'''

# codes of a chunk and of a stretch, tokens that a wave loads, tiles of a wave of the three kernels, workgroups that share rows of the down product
Rules = namedtuple("Rules", "chunk stretch tokens gemv gate_up down splits")
CHUNKS = [(4, 128), (4, 64), (4, 32), (2, 256), (2, 128), (2, 64), (8, 64), (8, 32)]   # (r, chunk)


@functools.lru_cache(maxsize=None)
def _lib():
    folder = tempfile.mkdtemp(prefix="grouped_plans_")
    src, lib = os.path.join(folder, "plans.cpp"), os.path.join(folder, "plans.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", CSRC, src, "-o", lib], check=True)
    out = ctypes.CDLL(lib)
    i64 = ctypes.c_int64
    out.grouped_rules.argtypes = [ctypes.c_int, i64, i64, i64, i64, i64, i64, ctypes.POINTER(i64)]
    return out


def rules(r, group, B=1, N=1, d=64, F=64, experts=1):
    """experts: as many as may be chosen, min(B top, E)."""
    out = (ctypes.c_int64 * 7)()
    _lib().grouped_rules(r, group, B, N, d, F, experts, out)
    return Rules(*out)


def products():
    """Sizes (r, group, B, N, K) for every form of the matrix-vector product: below and above the rows from which a wave takes two tiles, a whole
    number of rows neither of one tile nor of two, several stretches and the begin of one more; groups of a chunk, and of three."""
    cases = []
    for r, c in CHUNKS:
        for B, far in ((3, {2: 16384, 8: 16384, 4: 65536}[r]), (6, 8192), (13, 8192)):
            stretch = rules(r, c).stretch
            for N in (37, far + 21):
                if (r, c, B) == (4, 32, 3) and N > far:
                    continue   # (never two tiles)
                cases.append((r, c, B, N, 3 * stretch + c))
        cases.append((r, 3 * c, 2, 70, 15 * c))
    return cases


def layers():
    """Sizes (r, group, B, top, E, d, F) for every form of the layer's two products, rows ending inside a stretch and inside two tiles."""
    cases = []
    for r, c in CHUNKS:
        stretch, last = rules(r, c).stretch, max(c, 64)
        for B, top in ((3, 16), (7, 10), (13, 9)):
            E = 50                                # 48 or 50 experts
            few_f, many_f = last, -(-720 // last) * last
            few_d, many_d = last, -(-1472 // last) * last
            for d in (few_d, many_d):
                for F in (few_f, many_f):
                    cases.append((r, c, B, top, E, d, F))
        cases.append((r, c, 5, 2, 8, -(-8224 // c) * c, c))                       # enough rows for a workgroup's own down product
        cases.append((r, c, 1, 2, 4, last, 3 * c))                                # few pairs
        cases.append((r, c, 16, 16, 40, 2 * stretch + c, stretch + c))            # more pairs than waves
    return cases
