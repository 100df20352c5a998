"""Moves of tokens beyond the last-level cache, which are streamed, and blocks of 64 x 64 whose results are: against 64 bits, on the device, some tokens at a time.  The
bounds are those of test_gpu_experts and test_gpu_i8_products."""
import numpy as np
import pytest
import torch

import paper_2407_21418_amd as ft

from gpu_util import stream
from test_gpu_experts import TYPES, chain
from test_gpu_i8_kernels import spread
from test_gpu_i8_products import Output, Problem, check, check_gated
from test_operator_ranges import LARGE_RESULTS, STREAMED

pytestmark = pytest.mark.gpu

FORMS = [(s, d, odd) for s in STREAMED for d in (("f16", "bf16") if s[4] == 2 else ("f32",)) for odd in (False, True)]


class Large:
    """Rows in pitches of cols, or odd ones behind an odd offset; an entry in six has no row."""

    def __init__(self, tokens, top_k, experts, cols, dtype, odd):
        self.code, self.torch, self.rel, self.tiny = TYPES[dtype]
        self.tokens, self.top_k, self.cols, self.n = tokens, top_k, cols, tokens * top_k
        self.ld_token, self.ld_row, self.offset = (cols + 3, cols + 1, 1) if odd else (cols, cols, 0)
        self.gen = torch.Generator(device="cuda").manual_seed(tokens + cols)
        there = torch.rand(self.n, generator=self.gen, device="cuda") > 1 / 6
        rows = torch.randperm(self.n, generator=self.gen, device="cuda")                    # (rows that no entry has lie everywhere)
        self.row_of = torch.where(there, rows, -1).int()
        self.desc = ft.ft_expert_desc(experts=experts, top_k=top_k, cols=cols, ld_token=self.ld_token, ld_row=self.ld_row, dtype=self.code)
        self.used = torch.zeros(self.n, dtype=torch.bool, device="cuda")
        self.used[rows[there]] = True

    def buffer(self, count, pitch, fill=7.0):
        buf = torch.full((count * pitch + self.offset + 16,), fill, dtype=self.torch, device="cuda")
        return buf, buf[self.offset:self.offset + count * pitch].reshape(count, pitch)

    def random(self, count, pitch):
        buf, v = self.buffer(count, pitch, float("nan"))
        v[:, :self.cols] = torch.randn(count, self.cols, generator=self.gen, device="cuda").to(self.torch)
        return buf, v[:, :self.cols]

    def ptr(self, buf):
        return buf.data_ptr() + self.offset * buf.element_size()

    def taken(self, buf, whole, rows=None):
        torch.cuda.synchronize()
        assert bool((buf[:self.offset] == 7).all()) and bool((buf[self.offset + whole.numel():] == 7).all()) and bool((whole[:, self.cols:] == 7).all()), "write outside of the rows"
        if rows is not None:
            assert bool((whole[~rows] == 7).all()), "a row that no entry has"
        return whole[:, :self.cols]

    def slices(self):
        step = max(1, 4 * 10 ** 6 // (self.top_k * self.cols))
        for t in range(0, self.tokens, step):
            part = slice(t, min(self.tokens, t + step))
            r = self.row_of[part.start * self.top_k:part.stop * self.top_k].long().reshape(-1, self.top_k)
            yield part, r, r >= 0

    def entries(self, y, r):
        return torch.where((r >= 0)[:, :, None], y[r.clamp(min=0)].double(), torch.zeros((), dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("shape,dtype,odd", FORMS)
def test_moves(shape, dtype, odd):
    s = Large(*shape[:4], dtype, odd)
    xb, x = s.random(s.tokens, s.ld_token)
    yb, y = s.buffer(s.n, s.ld_row)
    ft.ft_expert_gather(s.desc, s.tokens, s.ptr(xb), s.row_of.data_ptr(), s.ptr(yb), stream())
    got = s.taken(yb, y, s.used)
    for part, r, there in s.slices():
        assert torch.equal(got[r[there]], x[part][:, None, :].expand(-1, s.top_k, -1)[there])
    del yb, y, got
    yb, y = s.random(s.n, s.ld_row)
    w = torch.rand(s.tokens, s.top_k, generator=s.gen, device="cuda") + 0.1
    w.reshape(-1)[s.row_of < 0] = float("nan")
    for weights in (w, None):
        at = weights.data_ptr() if weights is not None else 0
        ob, o = s.buffer(s.tokens, s.ld_token)
        ft.ft_expert_combine(s.desc, s.tokens, s.ptr(yb), s.row_of.data_ptr(), at, s.ptr(ob), stream())
        out = s.taken(ob, o)
        gb, g = s.buffer(s.n, s.ld_row)
        dw = torch.full((s.n + 2,), 7.0, device="cuda")
        ft.ft_expert_combine_grad(s.desc, s.tokens, s.ptr(xb), s.ptr(yb), s.row_of.data_ptr(), at, s.ptr(gb), dw.data_ptr() + 4, stream())
        dy = s.taken(gb, g, s.used)
        assert dw[0] == dw[-1] == 7
        for part, r, there in s.slices():
            w64 = torch.where(there, weights[part] if weights is not None else 1.0, 0.0).double()
            rows, d = s.entries(y, r), x[part].double()[:, None, :]
            terms = rows * w64[:, :, None]
            ref = terms.sum(1)
            assert bool(((out[part].double() - ref).abs() <= s.top_k * 2.0 ** -24 * terms.abs().sum(1) * 1.0001 + s.rel * ref.abs() * 1.0001 + s.tiny).all())
            ref = (w64[:, :, None] * d)[there]
            assert bool(((dy[r[there]].double() - ref).abs() <= (2.0 ** -24 + s.rel) * ref.abs() * 1.0001 + s.tiny).all())
            terms = rows * d
            off = (dw[1:-1].reshape(-1, s.top_k)[part].double() - terms.sum(2)).abs()
            assert bool((off <= chain(s.cols, s.code) * 2.0 ** -24 * terms.abs().sum(2) * 1.0001).all())
        gb2, g2 = s.buffer(s.n, s.ld_row)
        ft.ft_expert_combine_grad(s.desc, s.tokens, s.ptr(xb), 0, s.row_of.data_ptr(), at, s.ptr(gb2), 0, stream())
        assert torch.equal(s.taken(gb2, g2, s.used), dy)


@pytest.mark.parametrize("m,n,k,gates,experts", LARGE_RESULTS)
def test_blocks_of_64_with_large_results(m, n, k, gates, experts):
    weights, of_c = max(1, experts), n // 2 if gates else n
    p = Problem(3000 if experts else m, n, k, experts=weights, bias=not gates)
    if gates:
        p.sa /= k ** 0.5
    sizes = list(spread(m, experts)) if experts else [m]
    offsets = np.cumsum([0] + sizes)
    on_device = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    source = torch.randint(0, p.m, (m,), generator=torch.Generator().manual_seed(n)).cuda() if experts else torch.arange(m, device="cuda")
    a_row, bias = source.int(), p.bias.data_ptr() if p.bias is not None else 0
    for out in ("bf16", "f16", "f32"):
        c = Output(m, of_c, out)                             # (64 elements behind the buffer's beginning: rows on blocks of 64 bytes)
        args = (p.a.data_ptr(), p.sa.data_ptr())
        more = (p.b.data_ptr(), p.sb.data_ptr(), bias, c.ptr, stream())
        if experts:
            ft.ft_i8_matmul_experts(p.desc(out, 0, gates, experts=experts), m, on_device.data_ptr(), *args, a_row.data_ptr(), p.m, *more)
        else:
            ft.ft_i8_matmul(p.desc(out, 0, gates), m, *args, *more)
        got = c.take()
        for e in range(weights):
            rows = slice(int(offsets[e]), int(offsets[e + 1]))
            if rows.start < rows.stop:
                ref, size = p.exact(0, source[rows], e)
                if gates:
                    check_gated(got[rows], ref, out)
                else:
                    check(got[rows], ref, size, out)
