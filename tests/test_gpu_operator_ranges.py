"""Matmuls in 8-bit integers and moves of tokens where a launch's extents end: against exact integer sums and 64 bits."""
import pytest
import torch

import paper_2407_21418_amd as ft

from gpu_util import stream
from test_gpu_i8_kernels import check_product
from test_gpu_i8_products import Problem, check
from test_operator_ranges import ONE_ROW

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k,experts", ONE_ROW)
def test_blocks_of_one_row(m, n, k, experts):
    check_product(m, n, k, False, experts)


MOST_WORKGROUPS = (2 ** 32 - 1) // 256                       # of 256 threads in a launch


def test_more_rows_than_a_launch_quantises():
    """Four rows to a workgroup of 256 threads; every row against its definition (fp16 without an activation: exact)."""
    rows, cols, pitch = 4 * MOST_WORKGROUPS + 37, 5, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, cols, generator=gen, device="cuda", dtype=torch.float16)
    q, s = torch.full((rows, pitch), 77, dtype=torch.int8, device="cuda"), torch.full((rows,), -5.0, device="cuda")
    ft.ft_i8_quantize(ft.ft_quant_desc(cols=cols), rows, x.data_ptr(), q.data_ptr(), s.data_ptr(), stream())
    torch.cuda.synchronize()
    for at in range(0, rows, 1 << 23):
        part = slice(at, at + (1 << 23))
        f = x[part].double()
        peak = f.abs().amax(1, keepdim=True)
        want = torch.where(peak > 0, torch.round(127 * f / peak), torch.zeros_like(f))
        assert torch.equal(q[part, :cols].double(), want) and not bool(q[part, cols:].any()) and torch.equal(s[part], (peak[:, 0] / 127).float()), at


def test_more_tokens_than_a_launch_moves():
    """Rows of 129 pieces of 16 bytes take a workgroup a token.  Few tokens have a row: at both ends, and on both sides of where a launch ends."""
    tokens, top_k, cols = MOST_WORKGROUPS + 9, 2, 1025
    gen = torch.Generator(device="cuda").manual_seed(2)
    at = torch.tensor([0, 1, 77, MOST_WORKGROUPS - 2, MOST_WORKGROUPS - 1, MOST_WORKGROUPS, MOST_WORKGROUPS + 1, tokens - 1], device="cuda")
    rows = len(at) * top_k
    row_of = torch.full((tokens, top_k), -1, dtype=torch.int32, device="cuda")
    row_of[at] = torch.randperm(rows, generator=gen, device="cuda").reshape(-1, top_k).int()
    r = row_of[at].long()
    weights = torch.full((tokens, top_k), float("nan"), device="cuda")
    weights[at] = torch.rand(len(at), top_k, generator=gen, device="cuda") + 0.5
    half = dict(dtype=torch.bfloat16, device="cuda")
    token_rows = torch.empty(tokens, cols, **half)           # 34 GB: tokens to be read that no row asks for may hold anything
    token_rows[at] = torch.randn(len(at), cols, generator=gen, **half)
    y, dy = torch.full((rows + 1, cols), 7.0, **half), torch.full((rows + 1, cols), 7.0, **half)
    desc = ft.ft_expert_desc(experts=4, top_k=top_k, cols=cols, dtype=ft.FT_BF16)
    ft.ft_expert_gather(desc, tokens, token_rows.data_ptr(), row_of.data_ptr(), y.data_ptr(), stream())
    torch.cuda.synchronize()
    x = token_rows[at]
    assert torch.equal(y[r], x[:, None, :].expand(-1, top_k, -1)) and bool((y[rows] == 7).all())
    y[:rows] = torch.randn(rows, cols, generator=gen, **half)
    dweights = torch.full((tokens, top_k), 7.0, device="cuda")
    ft.ft_expert_combine_grad(desc, tokens, token_rows.data_ptr(), y.data_ptr(), row_of.data_ptr(), weights.data_ptr(), dy.data_ptr(), dweights.data_ptr(), stream())
    torch.cuda.synchronize()
    # (one product in fp32 and one rounding to bf16; sums of 1025 products in an order of at most 8 + 6 + 4 additions, see test_gpu_experts.chain)
    want = weights[at].double()[:, :, None] * x.double()[:, None, :]
    assert bool(((dy[r].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -24) * 1.0001 * want.abs()).all()) and bool((dy[rows] == 7).all())
    terms = y[r].double() * x.double()[:, None, :]
    assert bool(((dweights[at].double() - terms.sum(2)).abs() <= 18 * 2.0 ** -24 * 1.0001 * terms.abs().sum(2)).all())
    dweights[at] = 0
    assert not bool(dweights.any())
    out = token_rows.fill_(7.0)
    ft.ft_expert_combine(desc, tokens, y.data_ptr(), row_of.data_ptr(), weights.data_ptr(), out.data_ptr(), stream())
    torch.cuda.synchronize()
    terms = y[r].double() * weights[at].double()[:, :, None]
    ref = terms.sum(1)
    assert bool(((out[at].double() - ref).abs() <= 2 * 2.0 ** -24 * 1.0001 * terms.abs().sum(1) + 2.0 ** -8 * 1.0001 * ref.abs()).all())
    out[at] = 0
    assert not any(bool(out[a:a + (1 << 20)].any()) for a in range(0, tokens, 1 << 20))
    del token_rows, out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m,n,k,experts", [((1 << 27) + 33, 16, 16, 0), ((1 << 27) - 40, 16, 16, 3)])
def test_products_of_more_rows_than_threads_for_them(m, n, k, experts):
    a_rows = 1000 if experts else m
    p = Problem(a_rows, n, k, experts=max(1, experts), bias=True)
    c = torch.full((m + 1, n), 7.0, dtype=torch.float16, device="cuda")
    if experts:
        a_row = torch.randint(0, a_rows, (m,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda", dtype=torch.int32)
        offsets = [0, 1 << 26, 1 << 26, m]
        on_device = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        ft.ft_i8_matmul_experts(p.desc("f16", experts=experts), m, on_device.data_ptr(), p.a.data_ptr(), p.sa.data_ptr(), a_row.data_ptr(), a_rows, p.b.data_ptr(), p.sb.data_ptr(),
                                p.bias.data_ptr(), c.data_ptr(), stream())
    else:
        offsets = [0, m]
        ft.ft_i8_matmul(p.desc("f16"), m, p.a.data_ptr(), p.sa.data_ptr(), p.b.data_ptr(), p.sb.data_ptr(), p.bias.data_ptr(), c.data_ptr(), stream())
    torch.cuda.synchronize()
    assert bool((c[m] == 7).all())
    for e in range(max(1, experts)):
        for at in range(offsets[e], offsets[e + 1], 1 << 22):
            rows = slice(at, min(offsets[e + 1], at + (1 << 22)))
            ref, size = p.exact(0, a_row[rows].long() if experts else rows, e)
            check(c[rows], ref, size, "f16")


@pytest.mark.parametrize("rows,n", [(16, 80), (1300, 2064)])
def test_the_last_rows_of_2_gb(rows, n):
    """a_rows * lda just below 2^31: the last rows of A, and rows that it does not have."""
    lda, a_rows, k = 16384, 131071, 300
    p = Problem(1, n, k, experts=2)
    p.a, p.lda, p.sa = torch.zeros(a_rows, lda, dtype=torch.int8, device="cuda"), lda, torch.rand(a_rows, device="cuda") + 0.1
    p.a[-rows:] = torch.randint(-128, 128, (rows, lda), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda", dtype=torch.int8)
    source = torch.arange(a_rows - 1, a_rows - 1 - rows, -1, device="cuda")
    a_row = source.int()
    a_row[0], a_row[1] = a_rows, -1
    offsets = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    c = torch.full((rows, n), 7.0, device="cuda")
    ft.ft_i8_matmul_experts(p.desc("f32", experts=2), rows, offsets.data_ptr(), p.a.data_ptr(), p.sa.data_ptr(), a_row.data_ptr(), a_rows, p.b.data_ptr(), p.sb.data_ptr(), 0, c.data_ptr(), stream())
    torch.cuda.synchronize()
    for e, at in enumerate((slice(0, rows // 3), slice(rows // 3, rows))):
        ref, size = p.exact(0, source[at], e)
        if e == 0:
            ref[0], ref[1] = 0, 0
        check(c[at], ref, size, "f32")
