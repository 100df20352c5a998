"""Where matmuls in 8-bit integers and moves of tokens reach, by the rules of their launches compiled for the CPU (g++): copies that begin inside their rows,
launches that HIP takes, forms that large calls take."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

import paper_2407_21418_amd as ft

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "i8_blocks.h"
extern "C" int kernel(unsigned m, unsigned n, unsigned k, int gated, int experts) {
    ftk::I8Args a{};
    a.m = m; a.n = n; a.k = k; a.gated = gated; a.experts = experts; a.cus = 256;
    return (int)ftk::i8_choose(a, experts > 0);
}
extern "C" int streamed(unsigned entries, unsigned cols, unsigned bytes) {
    ftk::MoveArgs a{};
    a.entries = entries; a.cols = cols;
    return ftk::move_streams(a, bytes);
}
extern "C" unsigned most_rows(unsigned per, unsigned threads) { return ftk::launch_rows(per, threads); }
// the first turn whose scalar offset is at or beyond the reduce axis' end, or that reads other tiles than all of them once; -1: none
extern "C" int bad_turn(unsigned k, unsigned groups, unsigned xcd, int rotated) {
    const unsigned tiles = (k + 127u) / 128u, nk = (tiles + groups - 1u) / groups, whole = k / (128u * groups), first = rotated ? xcd * whole / 8u : 0u;
    static unsigned char seen[4096];
    for (unsigned i = 0; i < tiles; ++i) seen[i] = 0;
    for (unsigned t = 0; t < nk; ++t)
        for (unsigned g = 0; g < groups; ++g) {
            const unsigned begin = ftk::i8_turn_begin(t, groups, first, whole), at = begin + g * 128u;
            if (begin >= k || at % 128u) return (int)t;
            if (at < k && seen[at / 128u]++) return (int)t;
            if (t >= whole && begin != t * groups * 128u) return (int)t;          // (where the axis ends inside: the tiles that are cut)
        }
    for (unsigned i = 0; i < tiles; ++i)
        if (!seen[i]) return (int)nk;
    return -1;
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    at = tmp_path_factory.mktemp("ranges")
    (at / "rules.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2407_21418_amd", "csrc"), str(at / "rules.cpp"),
                    "-o", str(at / "rules.so")], check=True)
    return C.CDLL(str(at / "rules.so"))


@pytest.mark.parametrize("groups", [1, 2])
def test_copies_begin_inside_the_reduce_axis(rules, groups):
    """A tile of one row is read up to its pitch, k rounded up to 16 bytes, and a buffer's bound holds the lanes' offsets alone: the scalar one has to stay before it."""
    for k in list(range(1, 2100)) + [4096, 4100, 8191, 8192, 8193, 8300, 8449, 11008, 65537, 131071]:
        for xcd in range(8 if k >= 8192 else 1):
            assert rules.bad_turn(k, groups, xcd, int(k >= 8192)) == -1, (k, xcd)


# blocks of 64 x 64, two groups along the reduce axis, whose last rows and columns of blocks have one row or column, with an odd number of k-tiles: m, n, k, experts
ONE_ROW = [(65, 2049, 4100, 0), (129, 2049, 8310, 0), (33, 777, 4100, 7)]


def test_blocks_of_one_row(rules):
    for m, n, k, experts in ONE_ROW:
        assert rules.kernel(m, n, k, 0, experts) == 1 and (k + 127) // 128 % 2 == 1 and (experts or m % 64 == 1) and (n % 64 == 1 or experts), (m, n, k, experts)


@pytest.mark.parametrize("per,threads", [(4, 256), (1, 64), (1, 128), (1, 960), (1, 1024)] + [(256 // lanes, 256) for lanes in (8, 16, 32, 64, 128, 256)])
def test_launches_have_fewer_than_2_to_the_32_threads(rules, per, threads):
    most = rules.most_rows(per, threads) % (1 << 32)
    assert most % per == 0 and most // per * threads < 1 << 32 <= (most // per + 1) * threads


def test_the_first_kernel_s_launches_too(rules):
    """Its workgroups of 512 threads have a tile of 16 x 16 each, 16 x 32 with gates; the other kernels' take the tiles in turn."""
    for bits in range(20, 32):
        for m in (1 << bits) - 1, 5 << (bits - 3):
            if m >= 1 << 31:
                continue
            for n in [1 << b for b in range(20)] + [3, 17, 24, 48, 80, 1000, (1 << 20) - 2]:
                for k in (1, 128, 129, 512, 4096, 131071):
                    for gates in (0, 1):
                        if n % 2 and gates:
                            continue
                        for experts in (0, 1, 64, 1024):
                            tiles = (m // 16 + experts if experts else -(-m // 16)) * -(-n // (32 if gates else 16))
                            assert tiles * 512 < 1 << 32 or rules.kernel(m, n, k, gates, experts) > 0, (m, n, k, gates, experts)


@pytest.mark.parametrize("lda,a_rows,fits", [(16, (1 << 27) - 1, True), (16, 1 << 27, False), (16384, 131071, True), (16384, 131072, False), (1 << 20, 2047, True), (1 << 20, 2048, False)])
def test_rows_by_expert_lie_within_2_gb(lda, a_rows, fits):
    """a_rows * lda < 2^31 (no rows of C: nothing is launched)."""
    call = lambda: ft.ft_i8_matmul_experts(ft.ft_i8_desc(n=16, k=16, lda=lda, experts=2), 0, 0, 0, 0, 0, a_rows, 0, 0, 0, 0)  # noqa: E731
    if fits:
        return call()
    with pytest.raises(ft.FtError) as e:
        call()
    assert e.value.status == ft.FT_ERR_UNSUPPORTED


# tokens, top_k, experts, columns, bytes of a value: moves that are streamed
STREAMED = [(17000, 8, 16, 1001, 2), (8500, 8, 16, 1001, 4), (4100, 8, 60, 4097, 2), (2450000, 8, 5, 7, 2), (4200000, 32, 3, 1, 4), (33000, 2, 128, 2048, 2)]


def test_large_moves_are_streamed(rules):
    for tokens, top_k, _, cols, size in STREAMED:
        assert rules.streamed(tokens * top_k, cols, size), (tokens, cols)
    assert not rules.streamed(1 << 18, 512, 2) and rules.streamed((1 << 18) + 1, 512, 2)


# m, n, k, gates, experts: blocks of 64 x 64 whose results are 4 MB and more (in rows of whole blocks of 64 bytes they go through the L2) in 16 bits
LARGE_RESULTS = [(33001, 64, 3574, False, 0), (66001, 32, 2100, False, 0), (66001, 64, 2100, True, 0), (33001, 64, 3574, False, 5), (66001, 64, 2100, True, 5), (66001, 32, 2100, False, 40)]


def test_blocks_of_64_with_large_results(rules):
    for m, n, k, gates, experts in LARGE_RESULTS:
        assert rules.kernel(m, n, k, int(gates), experts) == 1, (m, n, k, gates, experts)
        assert 2 * m * (n // 2 if gates else n) >= 4 << 20
