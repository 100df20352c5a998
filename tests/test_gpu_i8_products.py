"""Matmuls in 8-bit integers, plain and by expert, against exact integer sums and 64 bits.

The sum is exact.  Its conversion to fp32, the two scales and the bias are at most four roundings, the last of the whole: |d| <= 3 * 2^-24 |p| +
2^-24 |p + b| <= 4 * 2^-24 (|p| + |b|), plus half a step of a 16-bit result."""
import numpy as np
import pytest
import torch

import paper_2407_21418_amd as ft

from gpu_util import stream

pytestmark = pytest.mark.gpu

OUTS = {"f32": (ft.FT_F16, ft.FT_OUT_F32, torch.float32, 0.0, 0.0), "f16": (ft.FT_F16, ft.FT_OUT_SAME, torch.float16, 2.0 ** -11, 2.0 ** -25),
        "bf16": (ft.FT_BF16, ft.FT_OUT_SAME, torch.bfloat16, 2.0 ** -8, 2.0 ** -134)}
GUARD = 64


def pitch(k):
    return (k + 15) // 16 * 16


def gated(p):
    """(silu(g) * u, how far fp32 may be from it) of products p = [g | u] in 64 bits.  g and u are within 3 * 2^-24 of themselves, which moves
    g / (1 + exp(-g)) by at most 1 + |g| times that; the activation itself is within 4 * 2^-23 (exp 2^-23, its sum 2^-24, the reciprocal 2^-23, two
    products 2^-23) and what the exponent -g log2 e loses: |g| log2 e 2^-24 by its rounding and 2^-26.2 |g| by that of log2 e (1.44269502 for
    1.44269504), times ln 2 in exp(-g), 1.22 |g| 2^-24 in all.  A gate below -88 leaves a zero."""
    g, u = p.chunk(2, dim=1)
    f = g / (1 + torch.exp(-g)) * u
    return f, 1.001 * f.abs() * (4 * 2.0 ** -23 + 1.25 * 2.0 ** -24 * g.abs() + 3 * 2.0 ** -24 * (2 + g.abs())) + 100 * np.exp(-87.0) * u.abs() + 2.0 ** -148


class Problem:
    def __init__(self, m, n, k, seed=0, experts=1, lda=0, ldb=0, bias=False, extreme=False):
        g = torch.Generator(device="cuda").manual_seed(seed + 31 * m + 7 * n + k)
        ints = lambda *s: torch.randint(-128, 128, s, generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
        self.m, self.n, self.k, self.experts = m, n, k, experts
        self.lda, self.ldb = lda or pitch(k), ldb or pitch(k)
        self.a, self.b = ints(m, self.lda), ints(experts * n, self.ldb)      # (padding holds integers too)
        if extreme:
            self.a[:], self.b[:] = -128, -128
        self.sa = torch.rand(m, generator=g, device="cuda") * 0.01 + 1e-4
        self.sb = torch.rand(experts * n, generator=g, device="cuda") * 0.01 + 1e-4
        self.bias = torch.randn(experts * n, generator=g, device="cuda") if bias else None

    def exact(self, rows, source, expert):
        """(C, |product| + |bias|) in 64 bits of rows of A `source` with the weight of `expert`."""
        at = slice(expert * self.n, (expert + 1) * self.n)
        p = self.a[source, :self.k].double() @ self.b[at, :self.k].double().t()
        assert p.numel() == 0 or float(p.abs().max()) < 2 ** 31
        p = p * self.sa[source].double()[:, None] * self.sb[at].double()[None, :]
        b = self.bias[at].double()[None, :] if self.bias is not None else torch.zeros(1, 1, dtype=torch.float64, device="cuda")
        return p + b, p.abs() + b.abs()

    def desc(self, out, ldc=0, gates=False, **more):
        dtype, out_dtype = OUTS[out][:2]
        return ft.ft_i8_desc(n=self.n, k=self.k, lda=self.lda, ldb=self.ldb, ldc=ldc, dtype=dtype, out_dtype=out_dtype,
                             epilogue=ft.FT_EPI_SILU_MUL if gates else ft.FT_EPI_BIAS if self.bias is not None else ft.FT_EPI_NONE, **more)


class Output:
    """C [m][ldc] of a type between canaries, `offset` elements behind a 16-byte boundary."""

    def __init__(self, m, n, out, ldc=0, offset=0):
        self.m, self.n, self.ldc, self.lo = m, n, ldc or n, GUARD + offset
        self.buf = torch.full((m * self.ldc + 2 * GUARD + offset,), 7.0, dtype=OUTS[out][2], device="cuda")
        self.ptr = self.buf.data_ptr() + self.lo * self.buf.element_size()

    def take(self):
        torch.cuda.synchronize()
        hi = self.lo + self.m * self.ldc
        assert bool((self.buf[:self.lo] == 7).all()) and bool((self.buf[hi:] == 7).all()), "write outside of C"
        c = self.buf[self.lo:hi].reshape(self.m, self.ldc)
        assert bool((c[:, self.n:] == 7).all()), "write between the rows of C"
        return c[:, :self.n]


def check(got, ref, size, out):
    rel, tiny = OUTS[out][3:]
    d = (got.double() - ref).abs()
    bound = 4.01 * 2.0 ** -24 * size + rel * ref.abs() * 1.0001 + tiny
    assert bool(torch.isfinite(got.float()).all()) and bool((d <= bound).all()), f"worst {float((d - bound).max())} over the bound"


def check_gated(got, p, out):
    f, bound = gated(p)
    rel, tiny = OUTS[out][3:]
    d = (got.double() - f).abs()
    assert bool((d <= bound * (1 + rel) + rel * f.abs() * 1.0001 + tiny).all()), f"worst {float((d - bound).max())} over the bound"


def run(p, out, ldc=0, offset=0):
    c = Output(p.m, p.n, out, ldc, offset)
    ft.ft_i8_matmul(p.desc(out, ldc), p.m, p.a.data_ptr(), p.sa.data_ptr(), p.b.data_ptr(), p.sb.data_ptr(), p.bias.data_ptr() if p.bias is not None else 0, c.ptr, stream())
    return c.take()


def check_plain(p, out, **kw):
    got = run(p, out, **kw)
    check(got, *p.exact(p.m, slice(None), 0), out)
    return got


SIZES = [(1, 1, 1), (1, 16, 16), (2, 3, 5), (16, 16, 64), (17, 33, 127), (15, 1000, 128), (1, 4096, 4096), (5, 777, 1000), (31, 130, 129), (33, 64, 300), (48, 48, 2000), (64, 64, 64), (65, 257, 191),
         (77, 768, 768), (100, 100, 1), (127, 300, 65), (128, 128, 128), (129, 129, 129), (200, 1024, 513), (256, 256, 256), (257, 511, 1025), (300, 2304, 768), (403, 1003, 1001), (512, 1, 4096),
         (640, 768, 640), (1000, 1000, 1000), (1025, 2049, 130), (2048, 16, 64), (1500, 4096, 1024), (4096, 4096, 256), (3000, 5000, 384)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_sizes(m, n, k):
    check_plain(Problem(m, n, k), ("f32", "f16", "bf16")[(m + n + k) % 3])


@pytest.mark.parametrize("out", OUTS)
@pytest.mark.parametrize("m,n,k", [(1, 100, 100), (20, 64, 257), (77, 768, 768), (259, 513, 400), (600, 1024, 1024)])
def test_types_bias_and_pitches(m, n, k, out):
    check_plain(Problem(m, n, k, bias=True), out)
    check_plain(Problem(m, n, k, seed=1, lda=pitch(k) + 48, ldb=pitch(k) + 16, bias=True), out, ldc=n + 3, offset=1)
    check_plain(Problem(m, n, k, seed=2), out, ldc=(n + 15) // 16 * 16)
    check_plain(Problem(m, n, k, seed=3), out, offset=3)


@pytest.mark.parametrize("out", OUTS)
@pytest.mark.parametrize("m,n,k", [(1, 2, 1), (1, 100, 100), (16, 32, 64), (20, 66, 257), (77, 1536, 768), (259, 514, 400), (600, 2048, 1024), (1100, 1430, 300), (2500, 3000, 520)])
def test_gates(m, n, k, out):
    p = Problem(m, n, k)
    p.sa /= k ** 0.5
    ref = p.exact(m, slice(None), 0)[0]
    for ldc, offset in ((0, 0), (n // 2 + 3, 1), ((n // 2 + 15) // 16 * 16, 0)):
        c = Output(m, n // 2, out, ldc, offset)
        ft.ft_i8_matmul(p.desc(out, ldc, gates=True), m, p.a.data_ptr(), p.sa.data_ptr(), p.b.data_ptr(), p.sb.data_ptr(), 0, c.ptr, stream())
        check_gated(c.take(), ref, out)


@pytest.mark.parametrize("m,n,k", [(3, 20, 131071), (130, 130, 131071), (300, 300, 65537)])
def test_the_largest_sums(m, n, k):
    p = Problem(m, n, k, extreme=True)
    check_plain(p, "f32")


def test_every_row_count():
    p = Problem(300, 96, 200, bias=True)
    ref, size = p.exact(300, slice(None), 0)
    for m in range(1, 301):
        c = Output(m, 96, "f32")
        ft.ft_i8_matmul(p.desc("f32"), m, p.a.data_ptr(), p.sa.data_ptr(), p.b.data_ptr(), p.sb.data_ptr(), p.bias.data_ptr(), c.ptr, stream())
        check(c.take(), ref[:m], size[:m], "f32")


def test_same_bits_twice_and_on_another_stream():
    p = Problem(500, 700, 900, bias=True)
    first = run(p, "f32").clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert torch.equal(run(p, "f32"), first)
    assert torch.equal(run(p, "f32", offset=4), first)


def test_scales_that_are_not_finite():
    p = Problem(40, 50, 60)
    p.sa[3], p.sa[7] = float("nan"), float("inf")
    p.sb[11] = float("nan")
    got = run(p, "f32")
    want = torch.isnan(p.sa)[:, None] | torch.isnan(p.sb)[None, :]
    assert torch.equal(torch.isnan(got) & ~torch.isinf(p.sa)[:, None], want & ~torch.isinf(p.sa)[:, None])
    assert bool((torch.isfinite(got) | want | torch.isinf(p.sa)[:, None]).all())


def test_results_far_apart():
    """Offsets of C beyond 32 bits."""
    p = Problem(1030, 300, 64)
    ldc = 1 << 22
    c = torch.full((p.m, ldc), 7.0, dtype=torch.float16, device="cuda")
    ft.ft_i8_matmul(p.desc("f16", ldc), p.m, p.a.data_ptr(), p.sa.data_ptr(), p.b.data_ptr(), p.sb.data_ptr(), 0, c.data_ptr(), stream())
    check(c[:, :300], *p.exact(p.m, slice(None), 0), "f16")
    assert bool((c[:, 300:400] == 7).all()) and bool((c[:, -100:] == 7).all())


# ---- by expert -----------------------------------------------------------------------------------


def run_grouped(p, sizes, out, gather, first=0, behind=0, bad=(), ldc=0, offset=0):
    """sizes: rows of each expert.  gather: rows of A in another order, some twice.  bad: (row, index) entries of a_row that name no row."""
    rows = first + sum(sizes) + behind
    offsets = torch.tensor(np.cumsum([first] + list(sizes)), dtype=torch.int32, device="cuda")
    source = torch.arange(rows, device="cuda") % p.m
    if gather:
        source = torch.randint(0, p.m, (rows,), generator=torch.Generator().manual_seed(rows)).cuda()
    a_row = source.to(torch.int32)
    for r, index in bad:
        a_row[r] = index
    c = Output(rows, p.n, out, ldc, offset)
    ft.ft_i8_matmul_experts(p.desc(out, ldc, experts=p.experts), rows, offsets.data_ptr(), p.a.data_ptr(), p.sa.data_ptr(), a_row.data_ptr() if gather else 0, p.m, p.b.data_ptr(), p.sb.data_ptr(),
                            p.bias.data_ptr() if p.bias is not None else 0, c.ptr, stream())
    got = c.take()
    assert bool((got[:first] == 7).all()) and bool((got[rows - behind:] == 7).all()), "rows that belong to no expert"
    none = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for r, _ in bad:
        none[r] = True
    at = first
    for e, n in enumerate(sizes):
        if n:
            ref, size = p.exact(n, source[at:at + n], e)
            b = p.bias[e * p.n:(e + 1) * p.n].double()[None, :] if p.bias is not None else 0.0
            lost = none[at:at + n, None]
            check(got[at:at + n], torch.where(lost, 0 * ref + b, ref), size, out)
        at += n
    return got


GROUPS = {"one": [5], "empty ones": [0, 3, 0, 0, 17, 0], "nothing": [0, 0, 0], "single rows": [1] * 40, "uneven": [300, 1, 0, 64, 129, 16, 33, 2], "all in one": [0, 0, 700, 0],
          "many": [i * 7 % 5 for i in range(130)], "1024": [1 if i % 100 == 3 else 0 for i in range(1024)], "large": [513, 256, 255, 1, 640, 128], "one more": [17] * 70}


@pytest.mark.parametrize("groups", GROUPS)
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("n,k", [(40, 100), (300, 272)])
def test_groups(groups, gather, n, k):
    sizes = GROUPS[groups]
    out = ("f32", "bf16", "f16")[len(sizes) % 3]
    p = Problem(max(1, sum(sizes)), n, k, experts=len(sizes), bias=len(sizes) % 2 == 0)
    run_grouped(p, sizes, out, gather)
    if gather:
        p = Problem(max(1, sum(sizes) // 4), n, k, seed=5, experts=len(sizes))
        run_grouped(p, sizes, out, True, ldc=n + 5, offset=1)


@pytest.mark.parametrize("groups", ["empty ones", "uneven", "many", "large"])
@pytest.mark.parametrize("n,k", [(42, 100), (300, 272)])
def test_groups_with_gates(groups, n, k):
    sizes = GROUPS[groups]
    p = Problem(sum(sizes), n, k, experts=len(sizes))
    p.sa /= k ** 0.5
    offsets = np.cumsum([0] + sizes)
    o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    c = Output(p.m, n // 2, "f32")
    ft.ft_i8_matmul_experts(p.desc("f32", gates=True, experts=p.experts), p.m, o.data_ptr(), p.a.data_ptr(), p.sa.data_ptr(), 0, p.m, p.b.data_ptr(), p.sb.data_ptr(), 0, c.ptr, stream())
    got = c.take()
    for e in range(len(sizes)):
        rows = slice(int(offsets[e]), int(offsets[e + 1]))
        check_gated(got[rows], p.exact(0, rows, e)[0], "f32")


@pytest.mark.parametrize("sizes", [[3, 0, 2], [100, 20, 300], [700, 800]])
def test_rows_of_no_expert_stay(sizes):
    p = Problem(first_rows(sizes), 130, 80, experts=len(sizes), bias=True)
    run_grouped(p, sizes, "f32", True, first=3, behind=70)
    run_grouped(p, sizes, "bf16", False, first=1, behind=5)


def first_rows(sizes):
    return sum(sizes) + 80


@pytest.mark.parametrize("sizes", [[2, 2], [200, 100], [900, 900]])
def test_rows_that_a_does_not_have_count_as_zeros(sizes):
    p = Problem(64, 100, 200, experts=2, bias=True)
    run_grouped(p, sizes, "f32", True, bad=[(0, -1), (2, 64), (3, 2 ** 31 - 1)])


@pytest.mark.parametrize("offsets", [[0, 10 ** 9, 10 ** 9, 10 ** 9], [-5, 20, 10, 400], [50, 40, 30, 20], [0, 100, 50, 100]])
def test_offsets_that_are_not_ascending_write_no_other_rows(offsets):
    p = Problem(100, 40, 64, experts=3)
    c = Output(100, 40, "f32")
    o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    ft.ft_i8_matmul_experts(p.desc("f32", experts=3), 100, o.data_ptr(), p.a.data_ptr(), p.sa.data_ptr(), 0, 100, p.b.data_ptr(), p.sb.data_ptr(), 0, c.ptr, stream())
    assert bool(torch.isfinite(c.take()).all())


def test_weights_far_apart():
    """Offsets of B beyond 32 bits: 70 weights of 64 MB each."""
    n, k, experts = 64, 1000, 70
    p = Problem(140, n, k, experts=1)
    ldb = 1 << 20
    b = torch.zeros(experts, n, ldb, dtype=torch.int8, device="cuda")
    last = torch.randint(-128, 128, (n, k), generator=torch.Generator().manual_seed(3), dtype=torch.int8).cuda()
    b[-1, :, :k] = last
    sb = p.sb.repeat(experts)
    offsets = (2 * torch.arange(experts + 1)).to(torch.int32).cuda()
    c = Output(140, n, "f32")
    ft.ft_i8_matmul_experts(ft.ft_i8_desc(n=n, k=k, ldb=ldb, experts=experts), 140, offsets.data_ptr(), p.a.data_ptr(), p.sa.data_ptr(), 0, 140, b.data_ptr(), sb.data_ptr(), 0, c.ptr, stream())
    got = c.take()
    assert not got[:-2].any()
    ref = (p.a[-2:, :k].double() @ last.double().t()) * p.sa[-2:].double()[:, None] * p.sb.double()[None, :]
    check(got[-2:], ref, ref.abs(), "f32")
