"""Gates far below zero, whose 1 + exp(-g) is near the largest fp32, with values that make their results matter.

1 + exp(-g) lies between 2^126 and 2^128 for g from -87.34 to -88.72: its reciprocal is below the smallest normal number, g / (1 + exp(-g)) is not.  The bounds are those of
test_gpu_quant_rows and test_gpu_i8_products -- 4 * 2^-23 and 1.25 |g| 2^-24 -- and 2^-22 for a reciprocal that is rounded to a subnormal number, whose step is 2^-149 for
2^-128 at least.  Below -88.73 exp(-g) is beyond fp32 and the result is a zero."""
import numpy as np
import pytest
import torch

import paper_2407_21418_amd as ft

from gpu_util import stream
from test_gpu_quant_rows import quantize

pytestmark = pytest.mark.gpu

GATES = [-60.0, -80.0, -86.5, -87.0, -87.25, -87.4, -87.5, -87.75, -88.0, -88.25, -88.5, -88.7]


def bound(g):
    return 1.001 * (4 * 2.0 ** -23 + 1.25 * 2.0 ** -24 * np.abs(g) + 2.0 ** -22)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [1e30, -3e38, 1.0])
def test_rows(dtype, value):
    """A row whose largest magnitude is such a gate's: its scale, and all of its integers."""
    x = torch.zeros(len(GATES), 10, dtype=dtype)
    x[:, 0], x[:, 5] = torch.tensor(GATES), value
    x[:, 1], x[:, 6] = torch.tensor(GATES), value / 4
    q, s = quantize(x, 5, ft.FT_ACT_SILU_MUL)
    g, u = x[:, :2].double().numpy(), x[:, 5:7].double().numpy()
    f = g / (1 + np.exp(-g)) * u
    peak = np.abs(f[:, 0])
    # (below 2^-100 the scale itself, or f, loses bits to subnormal steps of 2^-149)
    assert (np.abs(s - peak / 127) <= (bound(g[:, 0]) + 2.0 ** -24) * peak / 127 + 2.0 ** -148).all(), s
    if abs(value) > 1:
        assert (q[:, 0] == 127 * np.sign(f[:, 0])).all() and (np.abs(q[:, 1] - 127 * f[:, 1] / peak) <= 0.5 + 127 * (2 * bound(g[:, 0]) + 2.0 ** -23)).all() and not q[:, 2:].any()


@pytest.mark.parametrize("m", [3, 400, 3000])
@pytest.mark.parametrize("n", [2 * len(GATES), 2 * 72 * len(GATES)])
def test_products(m, n):
    """k = 1: a gate is -1 times its two scales, a value 1 times them; few rows and blocks through LDS."""
    half = n // 2
    a, b = torch.zeros(m, 16, dtype=torch.int8, device="cuda"), torch.zeros(n, 16, dtype=torch.int8, device="cuda")
    a[:, 0], b[:half, 0], b[half:, 0] = 1, -1, 1
    sa, sb = torch.ones(m, device="cuda"), torch.empty(n, device="cuda")
    sb[:half] = -torch.tensor(GATES, device="cuda").repeat(half // len(GATES))
    sb[half:] = torch.logspace(28, 38, half, device="cuda", dtype=torch.float64).float()
    c = torch.full((m, half), 7.0, device="cuda")
    ft.ft_i8_matmul(ft.ft_i8_desc(n=n, k=1, epilogue=ft.FT_EPI_SILU_MUL), m, a.data_ptr(), sa.data_ptr(), b.data_ptr(), sb.data_ptr(), 0, c.data_ptr(), stream())
    torch.cuda.synchronize()
    g, u = -sb[:half].double().cpu().numpy(), sb[half:].double().cpu().numpy()
    f = g / (1 + np.exp(-g)) * u
    assert (np.abs(c.double().cpu().numpy() - f) <= bound(g) * np.abs(f)).all()


def test_beyond_fp32_there_is_a_zero():
    x = torch.tensor([[-88.8, -200.0, -3e38, 1.0, 1e38, 1e38, 1e38, 1.0]])
    q, s = quantize(x, 4, ft.FT_ACT_SILU_MUL)
    assert list(q[0]) == [0, 0, 0, 127] and abs(s[0] * 127 - 0.7310585786) < 1e-6
