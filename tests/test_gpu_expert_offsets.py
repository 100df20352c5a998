"""Matmuls in 8-bit integers by expert whose offsets reach beyond the rows, or do not ascend: rows that no group claims stay as they were, groups that nothing overlaps are
products.  Few rows, and blocks through LDS."""
import pytest
import torch

import paper_2407_21418_amd as ft

from gpu_util import stream
from test_gpu_i8_products import Output, Problem, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,n,k", [(100, 40, 64), (1300, 2320, 300), (2600, 2064, 1100)])
@pytest.mark.parametrize("offsets,ascend", [([0, 9, 9, 9], True), ([-3, -2, 0.5, 9], True), ([-2 ** 31, 0, 0.25, 2 ** 31 - 1], True), ([0.2, 0.2, 0.7, 0.9], True), ([9, 9, 9, 9], True),
                                            ([-5, -4, -3, -2], True), ([0.5, 0.4, 0.3, 0.2], False), ([1, 0, -1, -2], False), ([0, 0.5, 0.2, 0.2], False), ([0.1, 0.8, 0.4, 0.6], False),
                                            ([0, 1, 0, 1], False)])
def test_offsets(rows, n, k, offsets, ascend):
    """offsets: fractions of the rows, and whole numbers beyond them as they are (9: nine times the rows)."""
    values = [int(v) if abs(v) > 2 ** 30 else int(v * rows) for v in offsets]
    p = Problem(rows, n, k, experts=3)
    c = Output(rows, n, "f32")
    o = torch.tensor(values, dtype=torch.int32, device="cuda")
    ft.ft_i8_matmul_experts(p.desc("f32", experts=3), rows, o.data_ptr(), p.a.data_ptr(), p.sa.data_ptr(), 0, rows, p.b.data_ptr(), p.sb.data_ptr(), 0, c.ptr, stream())
    got = c.take()
    held = [min(max(v, 0), rows) for v in values]
    groups = [range(a, max(a, b)) for a, b in zip(held, held[1:])]
    claimed = torch.zeros(rows, dtype=torch.int64, device="cuda")
    for g in groups:
        claimed[g.start:g.stop] += 1
    assert bool((got[claimed == 0] == 7).all()), "rows of no group"
    if ascend:
        for e, g in enumerate(groups):
            if len(g):
                ref, size = p.exact(0, slice(g.start, g.stop), e)
                check(got[g.start:g.stop], ref, size, "f32")
