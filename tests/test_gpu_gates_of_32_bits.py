"""Rows of 32-bit gates and values as 8-bit integers: the bounds of test_gpu_quant_rows.test_gated, whose inputs are exact here too."""
import numpy as np
import pytest
import torch

import paper_2407_21418_amd as ft

from test_gpu_quant_rows import quantize

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,ldx,offset", [(1, 1, 2, 0), (2, 9, 19, 1), (7, 715, 1430, 0), (3, 1408, 2816, 3), (300, 100, 208, 0), (1030, 513, 1026, 0), (2, 11008, 22016, 0), (2, 33001, 66002, 1)])
def test_gated(rows, cols, ldx, offset):
    x = 3 * torch.randn(rows, ldx, generator=torch.Generator().manual_seed(cols))
    q, s = quantize(x, cols, ft.FT_ACT_SILU_MUL, offset=offset)
    gate, up = x[:, :cols].double().numpy(), x[:, cols:2 * cols].double().numpy()
    f = gate / (1 + np.exp(-gate)) * up
    amax = np.abs(f).max(axis=1)
    off = (4 + 0.62 * np.abs(gate).max(axis=1)) * 2.0 ** -23
    assert (np.abs(s - amax / 127) <= (off + 2.0 ** -24) * 1.001 * amax / 127).all()
    assert (np.abs(q - 127 * f / amax[:, None]) <= 0.5 + 127 * (2 * off + 2.0 ** -23)[:, None]).all()


@pytest.mark.parametrize("at,value", [(0, float("nan")), (0, float("-inf")), (5, float("inf")), (6, float("nan")), (11, float("-inf"))])
def test_what_is_not_finite(at, value):
    x = torch.ones(2, 12)
    x[0, at] = value
    q, s = quantize(x, 6, ft.FT_ACT_SILU_MUL)
    assert np.isnan(s[0]) and not q[0].any() and np.isfinite(s[1]) and (q[1] == 127).all()
