"""Every kernel that a matmul in 8-bit integers can take, with one tile for a workgroup and with several, against exact integer sums and 64 bits: rows that
are written 16 bytes at a time and streamed, rows that are written value by value, blocks that rows, columns and the reduce axis end inside."""
import numpy as np
import pytest
import torch

import paper_2407_21418_amd as ft

from gpu_util import stream
from test_gpu_i8_products import Output, Problem, check, check_gated
from test_operator_kernels import CASES

pytestmark = pytest.mark.gpu


def spread(rows, experts):
    """Numbers of rows of the experts, some 0, their sum `rows`."""
    share = np.array([(i * 37 % 11) * (i % 5 != 1) for i in range(experts)], dtype=np.float64)
    sizes = np.floor(share / share.sum() * rows).astype(np.int64)
    sizes[2] += rows - sizes.sum()
    return sizes


@pytest.mark.parametrize("name,m,n,k,gates,experts", CASES)
def test_kernel(name, m, n, k, gates, experts):
    check_product(m, n, k, gates, experts)


# a reduce axis that every XCD goes through from another place on, ended inside a block, at its end and inside the last of two groups' blocks
@pytest.mark.parametrize("m,n,k,gates,experts", [(300, 776, 8191, False, 0), (300, 776, 8192, False, 0), (700, 1040, 9000, False, 0), (1300, 1040, 8449, False, 0), (300, 4112, 8200, True, 0),
                                                 (1030, 4112, 8320, False, 0), (770, 5136, 11008, True, 0), (2060, 4112, 9000, False, 0), (200, 1040, 8300, False, 7), (1000, 4112, 8192, True, 7),
                                                 (2570, 2064, 8200, False, 7)])
def test_long_reduce_axes(m, n, k, gates, experts):
    check_product(m, n, k, gates, experts)


def check_product(m, n, k, gates, experts):
    weights, of_c = max(1, experts), n // 2 if gates else n
    p = Problem(min(m, 3000) if experts else m, n, k, experts=weights, bias=not gates and m % 2 == 0)
    if gates:
        p.sa /= k ** 0.5
    if experts:
        offsets = np.cumsum([0] + list(spread(m, experts)))
        on_device = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        source = torch.randint(0, p.m, (m,), generator=torch.Generator().manual_seed(m + n)).cuda()
        a_row = source.to(torch.int32)
    got = []
    outs = [("f32", (of_c + 15) // 16 * 16, 0), ("bf16", (of_c + 31) // 32 * 32, 0), ("f16", of_c + 3, 1)]
    for out, ldc, offset in outs:
        c = Output(m, of_c, out, ldc, offset)
        bias = p.bias.data_ptr() if p.bias is not None else 0
        if experts:
            ft.ft_i8_matmul_experts(p.desc(out, ldc, gates, experts=experts), m, on_device.data_ptr(), p.a.data_ptr(), p.sa.data_ptr(), a_row.data_ptr(), p.m, p.b.data_ptr(), p.sb.data_ptr(), bias,
                                    c.ptr, stream())
        else:
            ft.ft_i8_matmul(p.desc(out, ldc, gates), m, p.a.data_ptr(), p.sa.data_ptr(), p.b.data_ptr(), p.sb.data_ptr(), bias, c.ptr, stream())
        got.append(c.take())
    for e in range(weights):
        lo, hi = (offsets[e], offsets[e + 1]) if experts else (0, m)
        for at in range(lo, hi, 4096):
            rows = slice(at, min(hi, at + 4096))
            ref, size = p.exact(rows.stop - at, source[rows] if experts else rows, e)
            for c, (out, _, _) in zip(got, outs):
                if gates:
                    check_gated(c[rows], ref, out)
                else:
                    check(c[rows], ref, size, out)
