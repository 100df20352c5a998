"""Which kernel a matmul in 8-bit integers takes: the rule, compiled for the CPU (g++), at sizes that reach every one of them.  CASES is what the tests on
a GPU run, so that no kernel goes without a result that was checked."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNELS = ["stream", "64x64", "64x128", "128x128", "128x256", "256x256"]
SOURCE = r"""
#include "i8_blocks.h"
extern "C" int choose(unsigned m, unsigned n, unsigned k, int gated, int experts) {
    ftk::I8Args a{};
    a.m = m; a.n = n; a.k = k; a.gated = gated; a.experts = experts; a.cus = 256;
    return (int)ftk::i8_choose(a, experts > 0);
}
extern "C" int grid(unsigned m, unsigned n, int kind, int gated, int experts, unsigned *rows, unsigned *cols) {
    ftk::I8Args a{};
    a.m = m; a.n = n; a.gated = gated; a.experts = experts;
    const ftk::I8KindInfo i = ftk::i8_kind_info((ftk::I8Kind)kind, gated != 0);
    const bool ok = ftk::i8_grid(a, i.tm, i.tn, experts > 0);
    *rows = a.row_tiles; *cols = a.col_tiles;
    return ok;
}
"""

# kernel, m, n, k, gates, experts (0: a plain product): one tile for a workgroup at most, and several
CASES = [
    ("stream", 33, 80, 65, False, 0), ("stream", 33, 2064, 65, False, 0), ("64x64", 33, 2064, 4100, False, 0), ("64x128", 1300, 264, 65, False, 0), ("128x128", 12300, 264, 65, False, 0),
    ("128x128", 1300, 6160, 65, False, 0), ("128x256", 2570, 8208, 4100, False, 0), ("256x256", 1025, 8208, 1100, False, 0), ("256x256", 3300, 8208, 520, False, 0),
    ("stream", 33, 80, 65, False, 7), ("stream", 33, 2064, 65, False, 7), ("64x64", 33, 776, 4100, False, 7), ("64x128", 33, 2320, 1100, False, 7), ("64x128", 1025, 6160, 65, False, 7),
    ("128x128", 517, 6160, 65, False, 7), ("128x128", 1300, 6160, 65, False, 7), ("128x256", 517, 8208, 2100, False, 7), ("128x256", 1300, 8208, 4100, False, 7),
    ("256x256", 2300, 3600, 1100, False, 7), ("256x256", 12300, 2064, 520, False, 7), ("stream", 33, 80, 65, False, 70), ("stream", 1025, 80, 65, False, 70),
    ("64x64", 33, 264, 2100, False, 70), ("64x128", 33, 776, 65, False, 70), ("64x128", 770, 5136, 65, False, 70), ("128x128", 5130, 528, 65, False, 70),
    ("128x128", 16390, 528, 65, False, 70), ("128x256", 5130, 2320, 6200, False, 70), ("stream", 33, 80, 65, True, 0), ("stream", 33, 2064, 65, True, 0), ("64x64", 1500, 80, 4100, True, 0),
    ("64x128", 130, 4112, 65, True, 0), ("128x128", 12300, 264, 65, True, 0), ("128x128", 1300, 6160, 65, True, 0), ("128x256", 2570, 8208, 4100, True, 0),
    ("256x256", 1025, 8208, 1100, True, 0), ("256x256", 3300, 8208, 520, True, 0), ("stream", 33, 80, 65, True, 7), ("stream", 33, 2064, 65, True, 7), ("64x64", 130, 776, 4100, True, 7),
    ("64x128", 33, 3600, 65, True, 7), ("64x128", 1025, 6160, 65, True, 7), ("128x128", 517, 6160, 65, True, 7), ("128x128", 1300, 6160, 65, True, 7), ("128x256", 517, 8208, 2100, True, 7),
    ("128x256", 1300, 8208, 4100, True, 7), ("256x256", 2300, 3600, 1100, True, 7), ("256x256", 12300, 2064, 520, True, 7), ("stream", 33, 80, 65, True, 70),
    ("stream", 1025, 80, 65, True, 70), ("64x64", 2300, 80, 300, True, 70), ("64x128", 33, 528, 65, True, 70), ("64x128", 770, 5136, 65, True, 70), ("128x128", 5130, 528, 65, True, 70),
    ("128x128", 16390, 528, 65, True, 70), ("128x256", 5130, 2320, 6200, True, 70),
    ("256x256", 66000, 2832, 2048, False, 70), ("256x256", 66000, 2832, 2048, True, 70)]


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    at = tmp_path_factory.mktemp("rule")
    (at / "rule.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2407_21418_amd", "csrc"), str(at / "rule.cpp"),
                    "-o", str(at / "rule.so")], check=True)
    return C.CDLL(str(at / "rule.so"))


def test_the_cases_reach_every_kernel(rule):
    for case in CASES:
        name, m, n, k, gates, experts = case
        assert KERNELS[rule.choose(m, n, k, int(gates), experts)] == name, case
    for gates in (False, True):
        for experts in (0, 7, 70):
            assert {c[0] for c in CASES if c[4:] == (gates, experts)} >= set(KERNELS), (gates, experts)


def test_a_choice_for_every_size(rule):
    rows, cols = C.c_uint32(), C.c_uint32()
    for m in (1, 2, 100, 4096, 1 << 20, (1 << 31) - 1):
        for n in (2, 130, 4096, (1 << 20) - 2):
            for k in (1, 128, 4096, 131071):
                for gates in (0, 1):
                    for experts in (0, 1, 64, 1024):
                        kind = rule.choose(m, n, k, gates, experts)
                        assert 0 <= kind < len(KERNELS)
                        if rule.grid(m, n, kind, gates, experts, C.byref(rows), C.byref(cols)):
                            assert rows.value * cols.value < 1 << 31
                        else:
                            assert m * n > 1 << 40
