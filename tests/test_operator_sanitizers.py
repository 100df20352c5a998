"""The argument checks of the operators, as the CPU build has them (host_stubs.cpp makes the library's own checks), under AddressSanitizer and UndefinedBehaviorSanitizer, and
the rule that chooses a product's kernel with conversions beyond their type caught as well."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2407_21418_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_refusals_under_asan_and_ubsan(tmp_path):
    asan = subprocess.run(["g++", "-print-file-name=libasan.so"], capture_output=True, text=True).stdout.strip()
    if not os.path.isabs(asan) or not os.path.exists(asan):
        pytest.skip("no libasan in this toolchain")
    lib = str(tmp_path / "libftuner_host_san.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fPIC", "-shared", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer",
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(CSRC, "host.cpp"), os.path.join(CSRC, "host_stubs.cpp"), "-o", lib], check=True)
    env = dict(os.environ, FTUNER_LIB=lib, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    # the sanitizer runtime has to come first among the preloaded libraries; whatever is preloaded already stays
    env["LD_PRELOAD"] = ":".join([asan] + [p for p in env.get("LD_PRELOAD", "").split(":") if p])
    p = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "tests/test_operator_refusals.py", "tests/test_native_operators.py"], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=600)
    tail = (p.stdout + p.stderr)[-3000:]
    assert p.returncode == 0 and "passed" in p.stdout and "ERROR: AddressSanitizer" not in tail and "runtime error" not in tail, tail


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_the_rule_under_ubsan(tmp_path):
    (tmp_path / "rule.cpp").write_text(r"""
#include "i8_blocks.h"
int main() {
    const unsigned m[] = {1, 16, 17, 4096, 1u << 20, 0x7fffffffu}, n[] = {2, 130, 4096, (1u << 20) - 2}, k[] = {1, 128, 4096, 131071}, experts[] = {0, 1, 64, 1024};
    unsigned sum = 0;
    for (unsigned a : m) for (unsigned b : n) for (unsigned c : k) for (unsigned e : experts) for (unsigned gated = 0; gated < 2; ++gated) {
        ftk::I8Args g{};
        g.m = a; g.n = b; g.k = c; g.gated = gated; g.experts = e; g.cus = 256;
        const ftk::I8Kind kind = ftk::i8_choose(g, e > 0);
        const ftk::I8KindInfo i = ftk::i8_kind_info(kind, gated != 0);
        sum += ftk::i8_grid(g, i.tm, i.tn, e > 0);
    }
    return sum == 0;
}
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=undefined,float-cast-overflow", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    str(tmp_path / "rule.cpp"), "-o", str(tmp_path / "rule")], check=True)
    p = subprocess.run([str(tmp_path / "rule")], capture_output=True, text=True, timeout=60)
    assert p.returncode == 0, p.stderr[-2000:]
