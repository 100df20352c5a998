"""Rows of values as 8-bit integers against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2407_21418_amd as ft

from gpu_util import stream

pytestmark = pytest.mark.gpu

TYPES = {ft.FT_F16: torch.float16, ft.FT_BF16: torch.bfloat16}
GUARD8 = 77


def quantize(x, cols, act=ft.FT_ACT_NONE, ldq=0, offset=0):
    """x: CPU tensor [rows, pitch].  Returns (integers [rows, cols], scales) after a look at the padding and at
    what lies around the outputs.  offset: elements between a 16-byte boundary and X."""
    rows, ldx = x.shape
    pitch = ldq or (cols + 15) // 16 * 16
    buf = torch.full((rows * ldx + offset + 8,), float("nan"), dtype=x.dtype, device="cuda")
    buf[offset:offset + rows * ldx] = x.reshape(-1).cuda()
    q = torch.full((rows * pitch + 32,), GUARD8, dtype=torch.int8, device="cuda")
    s = torch.full((rows + 2,), -5.0, device="cuda")
    dtype = {torch.float16: ft.FT_F16, torch.bfloat16: ft.FT_BF16, torch.float32: ft.FT_F32}[x.dtype]
    ft.ft_i8_quantize(ft.ft_quant_desc(cols=cols, ldx=ldx, ldq=ldq, dtype=dtype, act=act), rows, buf.data_ptr() + x.element_size() * offset, q.data_ptr() + 16, s.data_ptr() + 4, stream())
    torch.cuda.synchronize()
    q, s = q.cpu().numpy(), s.cpu().numpy()
    assert (q[:16] == GUARD8).all() and (q[16 + rows * pitch:] == GUARD8).all() and s[0] == s[-1] == -5.0, "write outside of the outputs"
    q = q[16:16 + rows * pitch].reshape(rows, pitch)
    assert (q[:, cols:] == 0).all(), "padding"
    return q[:, :cols].astype(np.float64), s[1:-1]


def check_exact(x, cols, **kw):
    q, s = quantize(x, cols, **kw)
    f = x[:, :cols].double().numpy()
    amax = np.abs(f).max(axis=1)
    assert np.array_equal(s, amax.astype(np.float32) / np.float32(127))
    # (64 bits separate every quotient of 16-bit values from the middle between two integers, and represent the middles)
    want = np.rint(127 * f / np.where(amax == 0, 1, amax)[:, None])
    assert np.array_equal(q, want), f"{(q != want).sum()} of {q.size} integers differ"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 17), (1, 4096), (9, 511), (9, 512), (9, 513), (4, 1024), (3, 1025), (2, 8191), (2, 11008), (2, 16384), (2, 16385), (2, 32768), (2, 32769),
                                       (1, 70001), (1030, 64)])
def test_against_the_definition(dtype, rows, cols):
    g = torch.Generator().manual_seed(rows * 7919 + cols)
    check_exact(torch.randn(rows, cols, generator=g).to(TYPES[dtype]), cols)


@pytest.mark.parametrize("dtype", TYPES)
def test_middles_between_two_integers(dtype):
    """Every value of a type's significand against every peak: the quotients that lie in the middle, and those next to it."""
    bits = 11 if dtype == ft.FT_F16 else 8
    a = torch.arange(1, 2 ** bits, dtype=torch.float32)
    peaks = torch.cat([torch.arange(2 ** (bits - 1), 2 ** bits, max(1, 2 ** bits // 512)), torch.tensor([2 ** bits - 1, 2 ** (bits - 1), 127, 254])]).float()
    x = torch.cat([a, -a, a / 16, a / 256]).to(TYPES[dtype]).repeat(len(peaks), 1)
    x = torch.where(x.float().abs() <= peaks[:, None], x, torch.zeros_like(x))
    x[:, 0] = peaks.to(TYPES[dtype])
    check_exact(x, x.shape[1])


@pytest.mark.parametrize("offset,extra", [(0, 0), (1, 0), (3, 5), (0, 8), (7, 1)])
def test_pitches_and_alignment(offset, extra):
    x = torch.randn(6, 200 + extra, generator=torch.Generator().manual_seed(offset)).to(torch.float16)
    x[:, 200:] = float("inf")
    check_exact(x, 200, offset=offset)
    check_exact(x, 200, offset=offset, ldq=304)
    check_exact(x[:, :197].contiguous(), 197, offset=offset)


@pytest.mark.parametrize("dtype", TYPES)
def test_extreme_rows(dtype):
    t = TYPES[dtype]
    tiny, most = torch.finfo(t).smallest_normal, torch.finfo(t).max
    sub = tiny * torch.finfo(t).eps                          # the smallest subnormal
    x = torch.zeros(8, 40, dtype=t)
    x[1, 3] = sub
    x[2] = torch.arange(40).to(t) * sub
    x[3] = most
    x[4, ::2] = -most
    x[5, 7] = tiny
    x[6] = torch.linspace(-1, 1, 40).to(t) * tiny
    x[7, 39] = -1.0
    check_exact(x, 40)
    q, s = quantize(x, 40)
    assert s[0] == 0 and (q[0] == 0).all() and q[1, 3] == 127 and q[7, 39] == -127


@pytest.mark.parametrize("act", [ft.FT_ACT_NONE, ft.FT_ACT_SILU_MUL])
@pytest.mark.parametrize("cols", [5, 600, 33000])
def test_infinities_and_nans_are_not_lost(act, cols):
    width = cols if act == ft.FT_ACT_NONE else 2 * cols
    x = torch.ones(6, width, dtype=torch.bfloat16)
    for r, v in enumerate((float("inf"), float("-inf"), float("nan"), -float("nan"))):
        x[r, (r * 977) % width] = v
    x[4, width - 1] = float("nan")
    q, s = quantize(x, cols, act)
    assert np.isnan(s[:5]).all() and (q[:5] == 0).all() and np.isfinite(s[5]) and (q[5] == 127).all()


@pytest.mark.parametrize("rows,cols,extra,offset", [(1, 1, 0, 0), (5, 17, 2, 1), (9, 511, 0, 3), (3, 1025, 7, 0), (2, 16385, 0, 0), (2, 33001, 3, 1)])
def test_32_bits(rows, cols, extra, offset):
    """The quotient is rounded once, 2^-24 of itself (the second part of 127 / amax leaves 2^-46): half a step and 127 * 2^-23 in all."""
    x = torch.randn(rows, cols + extra, generator=torch.Generator().manual_seed(cols))
    x[0] *= 1e-38
    q, s = quantize(x, cols, offset=offset)
    f = x[:, :cols].double().numpy()
    amax = np.abs(f).max(axis=1)
    assert np.array_equal(s, (amax / 127).astype(np.float32))
    assert (np.abs(q - 127 * f / amax[:, None]) <= 0.5 + 127 * 2.0 ** -23).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,ldx", [(1, 1, 2), (2, 9, 19), (7, 715, 1430), (3, 1408, 2816), (2, 11008, 22016), (2, 33001, 66002), (300, 100, 208)])
def test_gated(dtype, rows, cols, ldx):
    """f in fp32: exp within 2^-23 of itself, 1 + exp 2^-24, the reciprocal 2^-23, two products 2^-23: less than 4 * 2^-23 in all; and what the
    exponent -g log2 e loses, 1.22 |g| 2^-24 in exp(-g) (see test_gpu_i8_products).  Twice that for f / amax, and 2^-23 for the
    rounding of the quotient: an integer is at most half a step and 127 times that away."""
    g = torch.Generator().manual_seed(cols)
    x = (3 * torch.randn(rows, ldx, generator=g)).to(TYPES[dtype])
    q, s = quantize(x, cols, ft.FT_ACT_SILU_MUL)
    gate, up = x[:, :cols].double().numpy(), x[:, cols:2 * cols].double().numpy()
    f = gate / (1 + np.exp(-gate)) * up
    amax = np.abs(f).max(axis=1)
    off = (4 + 0.62 * np.abs(gate).max(axis=1)) * 2.0 ** -23
    assert (np.abs(s - amax / 127) <= (off + 2.0 ** -24) * 1.001 * amax / 127).all()
    assert (np.abs(q - 127 * f / amax[:, None]) <= 0.5 + 127 * (2 * off + 2.0 ** -23)[:, None]).all()


def test_gates_far_out():
    x = torch.tensor([[-1000.0, -90.0, 90.0, 1000.0, 0.0, -0.0, 2.0, 3.0, 1.0, 1.0, 1.0, 1.0]], dtype=torch.bfloat16)
    q, s = quantize(x, 6, ft.FT_ACT_SILU_MUL)                # gates and their factors: all finite, the peak is 1000 * 1
    assert s[0] == np.float32(1000) / np.float32(127) and list(q[0]) == [0, 0, 11, 127, 0, 0]


def test_rows_far_apart():
    """Offsets beyond 32 bits: the last rows of a buffer of 4.3 GB."""
    cols, ldx = 1000, 1 << 21
    rows = (1 << 31) // ldx + 3
    x = torch.zeros(rows, ldx, dtype=torch.float16, device="cuda")
    x[-2:, :cols] = torch.randn(2, cols, generator=torch.Generator().manual_seed(1)).to(torch.float16).cuda()
    q = torch.zeros(rows, 1008, dtype=torch.int8, device="cuda")
    s = torch.zeros(rows, device="cuda")
    ft.ft_i8_quantize(ft.ft_quant_desc(cols=cols, ldx=ldx), rows, x.data_ptr(), q.data_ptr(), s.data_ptr(), stream())
    want, ws = quantize(x[-2:, :cols].cpu().contiguous(), cols)
    assert np.array_equal(q[-2:, :cols].cpu().numpy(), want) and np.array_equal(s[-2:].cpu().numpy(), ws) and not q[:-2].any() and not s[:-2].any()
