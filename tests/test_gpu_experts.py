"""Tokens sorted by expert and back, and the gradients, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2407_21418_amd as ft

from gpu_util import stream

pytestmark = pytest.mark.gpu

TYPES = {"f16": (ft.FT_F16, torch.float16, 2.0 ** -11, 2.0 ** -25), "bf16": (ft.FT_BF16, torch.bfloat16, 2.0 ** -8, 2.0 ** -134), "f32": (ft.FT_F32, torch.float32, 2.0 ** -24, 2.0 ** -150)}


def route(ids, experts):
    """ids [tokens, top_k] (numpy) -> offsets, row_token, row_of."""
    flat = ids.reshape(-1)
    kept = np.flatnonzero((flat >= 0) & (flat < experts))
    order = kept[np.argsort(flat[kept], kind="stable")]
    row_of = np.full(flat.size, -1)
    row_of[order] = np.arange(order.size)
    row_token = np.full(flat.size, -1)
    row_token[:order.size] = order // ids.shape[1]
    return np.searchsorted(flat[order], np.arange(experts + 1)), row_token, row_of


def sort(ids, experts, workspace=None):
    tokens, top_k = ids.shape
    desc = ft.ft_expert_desc(experts=experts, top_k=top_k)
    n = tokens * top_k
    need = ft.ft_expert_workspace(desc, tokens)
    ws = workspace if workspace is not None else torch.randint(0, 255, (need + 64,), dtype=torch.uint8, device="cuda")
    d = torch.from_numpy(ids.astype(np.int32)).cuda()
    outs = [torch.full((size + 8,), -77, dtype=torch.int32, device="cuda") for size in (experts + 1, n, n)]
    ft.ft_expert_sort(desc, tokens, d.data_ptr(), *(o.data_ptr() + 16 for o in outs), ws.data_ptr(), need, stream())
    torch.cuda.synchronize()
    for o in outs:
        assert bool((o[:4] == -77).all()) and bool((o[-4:] == -77).all()), "write outside of the outputs"
    assert workspace is not None or need == 0 or ws.numel() == need + 64
    return [o[4:-4].cpu().numpy() for o in outs]


def check_sort(ids, experts):
    for got, want in zip(sort(ids, experts), route(ids, experts)):
        assert np.array_equal(got, want)


@pytest.mark.parametrize("tokens,top_k,experts", [(0, 2, 8), (1, 1, 1), (1, 8, 8), (5, 2, 8), (63, 1, 4), (64, 1, 64), (65, 1, 65), (33, 2, 1), (1000, 2, 16), (1234, 6, 60), (700, 3, 1024), (4096, 2, 128),
                                                  (4097, 2, 128), (8191, 1, 7), (8192, 8, 128), (5000, 7, 1000), (1, 32, 1024), (100000, 8, 256), (300001, 5, 3)])
@pytest.mark.parametrize("dropped", [0.0, 0.3])
def test_sort(tokens, top_k, experts, dropped):
    g = np.random.default_rng(tokens + experts)
    ids = g.integers(0, experts, size=(tokens, top_k))
    ids[g.random(ids.shape) < dropped] = -1
    check_sort(ids, experts)


def test_sort_of_uneven_and_odd_ids():
    g = np.random.default_rng(1)
    check_sort(np.full((3000, 4), 5), 8)                     # everything to one expert
    check_sort(np.full((3000, 4), -1), 8)                    # nothing to any
    check_sort(g.choice([7, 8, -1, 2 ** 31 - 1, -2 ** 31, 0], size=(5000, 3)), 8)       # ids beyond the last expert
    check_sort(np.sort(g.integers(0, 50, size=20000))[:, None], 50)
    check_sort(np.sort(g.integers(0, 50, size=20000))[::-1].copy()[:, None], 50)
    check_sort(np.repeat(g.integers(0, 9, size=(999, 1)), 6, axis=1), 9)                # the same expert several times


class Moves:
    def __init__(self, tokens, top_k, experts, cols, dtype, dropped=0.2, ld_token=0, ld_row=0, seed=0, offset=0):
        self.code, self.torch, self.rel, self.tiny = TYPES[dtype]
        g = np.random.default_rng(seed + tokens + cols)
        ids = g.integers(0, experts, size=(tokens, top_k))
        ids[g.random(ids.shape) < dropped] = -1
        self.tokens, self.top_k, self.cols, self.n = tokens, top_k, cols, tokens * top_k
        self.ld_token, self.ld_row, self.offset = ld_token or cols, ld_row or cols, offset
        self.row_of = torch.from_numpy(route(ids, experts)[2].astype(np.int32)).cuda()
        self.gen = torch.Generator().manual_seed(seed + cols)
        self.desc = ft.ft_expert_desc(experts=experts, top_k=top_k, cols=cols, ld_token=ld_token, ld_row=ld_row, dtype=self.code)

    def rows(self, count, pitch):
        """Random rows `offset` elements behind a boundary, NaN in whatever is not theirs."""
        buf = torch.full((count * pitch + self.offset + 16,), float("nan"), dtype=self.torch, device="cuda")
        v = buf[self.offset:self.offset + count * pitch].reshape(count, pitch)[:, :self.cols]
        v.copy_(torch.randn(count, self.cols, generator=self.gen).to(self.torch))
        return buf, v

    def output(self, count, pitch):
        buf = torch.full((count * pitch + self.offset + 16,), 7.0, dtype=self.torch, device="cuda")
        return buf, buf[self.offset:self.offset + count * pitch].reshape(count, pitch)

    def ptr(self, buf):
        return buf.data_ptr() + self.offset * buf.element_size()

    def taken(self, buf, whole, rows):
        """The output's rows; whatever else is in the buffer has to be as it was.  rows: truth value for each row that is written."""
        torch.cuda.synchronize()
        assert bool((buf[:self.offset] == 7).all()) and bool((buf[self.offset + whole.numel():] == 7).all()) and bool((whole[:, self.cols:] == 7).all()), "write outside of the rows"
        assert bool((whole[~rows] == 7).all()), "a row that no entry has"
        return whole[:, :self.cols].double().cpu()

    @property
    def used(self):
        u = torch.zeros(self.n, dtype=torch.bool, device="cuda")
        u[self.row_of[self.row_of >= 0].long()] = True
        return u

    def entries(self, y):
        """[tokens, top_k, cols] in 64 bits, zeros where an entry has no row."""
        r = self.row_of.cpu().long()
        got = y.double().cpu()[r.clamp(min=0)]
        return torch.where((r >= 0)[:, None], got, torch.zeros((), dtype=torch.float64)).reshape(self.tokens, self.top_k, self.cols)

    def weights(self):
        w = torch.rand(self.tokens, self.top_k, generator=self.gen) + 0.1
        w.reshape(-1)[self.row_of.cpu() < 0] = float("nan")   # the weight of an entry without a row is nobody's
        return w.cuda(), torch.where(torch.isnan(w), torch.zeros(()), w).double()


SHAPES = [(1, 1, 1, 1), (1, 2, 4, 64), (5, 2, 8, 1024), (3, 8, 8, 7), (7, 3, 5, 9), (64, 9, 16, 100), (33, 17, 40, 250), (10, 32, 64, 65), (100, 8, 16, 513), (1234, 6, 60, 1001), (300, 4, 4, 2048), (50, 2, 8, 4097),
          (9, 5, 6, 20000)]


@pytest.mark.parametrize("tokens,top_k,experts,cols", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_gather(tokens, top_k, experts, cols, dtype):
    for kw in ({}, dict(ld_token=cols + 3, ld_row=cols + 1, offset=1), dict(ld_token=(cols + 7) // 8 * 8, ld_row=(cols + 15) // 8 * 8)):
        s = Moves(tokens, top_k, experts, cols, dtype, **kw)
        xb, x = s.rows(tokens, s.ld_token)
        yb, y = s.output(s.n, s.ld_row)
        ft.ft_expert_gather(s.desc, tokens, s.ptr(xb), s.row_of.data_ptr(), s.ptr(yb), stream())
        got = s.taken(yb, y, s.used)
        r = s.row_of.cpu().long()
        want = x.double().cpu().repeat_interleave(top_k, dim=0)
        assert torch.equal(got[r[r >= 0]], want[r >= 0])


@pytest.mark.parametrize("tokens,top_k,experts,cols", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("weighted", [True, False])
def test_combine(tokens, top_k, experts, cols, dtype, weighted):
    """top_k fused multiply-adds: each rounding is at most 2^-24 of the sum of magnitudes so far; then one to the type."""
    for kw in ({}, dict(ld_token=cols + 3, ld_row=cols + 1, offset=1)):
        s = Moves(tokens, top_k, experts, cols, dtype, **kw)
        yb, y = s.rows(s.n, s.ld_row)
        ob, o = s.output(tokens, s.ld_token)
        w, w64 = s.weights()
        if not weighted:
            w64 = torch.ones_like(w64)
        ft.ft_expert_combine(s.desc, tokens, s.ptr(yb), s.row_of.data_ptr(), w.data_ptr() if weighted else 0, s.ptr(ob), stream())
        got = s.taken(ob, o, torch.ones(tokens, dtype=torch.bool, device="cuda"))
        terms = s.entries(y) * w64[:, :, None]
        ref = terms.sum(dim=1)
        bound = top_k * 2.0 ** -24 * terms.abs().sum(dim=1) * 1.0001 + s.rel * ref.abs() * 1.0001 + s.tiny
        assert bool(((got - ref).abs() <= bound).all())


def chain(cols, code):
    """Additions in a row behind one another in a sum over the columns: those of a thread, then over the threads and the waves."""
    v = 4 if code == ft.FT_F32 else 8
    pieces = -(-cols // v)
    lanes = 8
    while lanes < 256 and lanes < pieces:
        lanes *= 2
    return -(-pieces // lanes) * v + 6 + 4


@pytest.mark.parametrize("tokens,top_k,experts,cols", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("weighted", [True, False])
def test_gradients(tokens, top_k, experts, cols, dtype, weighted):
    for kw in ({}, dict(ld_token=cols + 3, ld_row=cols + 1, offset=1)):
        s = Moves(tokens, top_k, experts, cols, dtype, **kw)
        yb, y = s.rows(s.n, s.ld_row)
        db, dout = s.rows(tokens, s.ld_token)
        w, w64 = s.weights()
        if not weighted:
            w64 = torch.ones_like(w64)
        gb, dy = s.output(s.n, s.ld_row)
        dw = torch.full((s.n + 2,), 7.0, device="cuda")
        args = (s.desc, tokens, s.ptr(db))
        more = (s.row_of.data_ptr(), w.data_ptr() if weighted else 0)
        ft.ft_expert_combine_grad(*args, s.ptr(yb), *more, s.ptr(gb), dw.data_ptr() + 4, stream())
        got = s.taken(gb, dy, s.used)
        r = s.row_of.cpu().long()
        d64 = dout.double().cpu()
        ref = (d64[:, None, :] * w64[:, :, None]).reshape(s.n, cols)[r >= 0]
        assert bool(((got[r[r >= 0]] - ref).abs() <= (2.0 ** -24 + s.rel) * ref.abs() * 1.0001 + s.tiny).all())
        terms = s.entries(y) * d64[:, None, :]
        assert dw[0] == dw[-1] == 7
        off = (dw[1:-1].double().cpu().reshape(tokens, top_k) - terms.sum(dim=2)).abs()
        assert bool((off <= chain(cols, s.code) * 2.0 ** -24 * terms.abs().sum(dim=2) * 1.0001).all())
        # without the weights' gradient Y is not looked at, and dY is the same
        gb2, dy2 = s.output(s.n, s.ld_row)
        ft.ft_expert_combine_grad(*args, 0, *more, s.ptr(gb2), 0, stream())
        assert torch.equal(s.taken(gb2, dy2, s.used), got)


def test_gradients_against_differences():
    """L = <dOut, combine(Y, w)> is linear in Y and in w: its differences are its gradient, up to the roundings of the two values of
    combine (fp32 rows: at most 4 * 2^-24 of the sum of magnitudes in each of 96 columns) over the step."""
    s = Moves(6, 3, 4, 96, "f32", dropped=0.25)
    yb, y = s.rows(s.n, s.ld_row)
    db, dout = s.rows(6, s.ld_token)
    w, w64 = s.weights()
    gb, dy = s.output(s.n, s.ld_row)
    dw = torch.zeros(s.n, device="cuda")
    ft.ft_expert_combine_grad(s.desc, 6, s.ptr(db), s.ptr(yb), s.row_of.data_ptr(), w.data_ptr(), s.ptr(gb), dw.data_ptr(), stream())

    def loss():
        ob, o = s.output(6, s.ld_token)
        ft.ft_expert_combine(s.desc, 6, s.ptr(yb), s.row_of.data_ptr(), w.data_ptr(), s.ptr(ob), stream())
        torch.cuda.synchronize()
        return float((o[:, :96].double() * dout.double()).sum())

    rows = s.row_of.cpu().tolist()
    size = float((s.entries(y).abs() * w64[:, :, None] * dout.double().cpu().abs()[:, None, :]).sum())
    h = 0.5                                                  # (powers of two: the step itself is exact up to one rounding of the value)
    for entry in range(s.n):
        if rows[entry] < 0:
            assert dw[entry] == 0
            continue
        base = loss()
        old = w.reshape(-1)[entry].clone()
        w.reshape(-1)[entry] += h
        step = float(w.reshape(-1)[entry]) - float(old)
        assert abs((loss() - base) / step - float(dw[entry])) <= 2 * 5 * 2.0 ** -24 * 2 * size / h
        w.reshape(-1)[entry] = old
        r, c = rows[entry], entry * 11 % 96
        old = y[r, c].clone()
        y[r, c] += h
        step = float(y[r, c]) - float(old)
        assert abs((loss() - base) / step - float(dy[r, c])) <= 2 * 5 * 2.0 ** -24 * 2 * size / h
        y[r, c] = old


def test_rows_that_are_not_there_are_none():
    s = Moves(4, 2, 4, 32, "f32", dropped=0.0)
    s.row_of[1], s.row_of[4], s.row_of[6] = 8, -2 ** 31, 2 ** 31 - 1          # outside of 0 .. 7
    gone = torch.tensor([1, 4, 6])
    xb, x = s.rows(4, 32)
    yb, y = s.output(8, 32)
    ft.ft_expert_gather(s.desc, 4, s.ptr(xb), s.row_of.data_ptr(), s.ptr(yb), stream())
    ob, o = s.output(4, 32)
    ft.ft_expert_combine(s.desc, 4, s.ptr(yb), s.row_of.data_ptr(), 0, s.ptr(ob), stream())
    torch.cuda.synchronize()
    count = torch.full((8,), 1.0)
    count[gone] = 0
    assert torch.equal(o.cpu(), x.cpu() * count.reshape(4, 2).sum(dim=1)[:, None])


def test_rows_far_apart():
    """Offsets beyond 32 bits, in both layouts."""
    pitch = 1 << 22
    s = Moves(520, 1, 2, 100, "bf16", dropped=0.0, ld_token=pitch, ld_row=pitch)
    x = torch.zeros(520, pitch, dtype=torch.bfloat16, device="cuda")
    x[:, :100] = torch.randn(520, 100, generator=s.gen).to(torch.bfloat16).cuda()
    y = torch.zeros(520, pitch, dtype=torch.bfloat16, device="cuda")
    back = torch.zeros_like(x)
    ft.ft_expert_gather(s.desc, 520, x.data_ptr(), s.row_of.data_ptr(), y.data_ptr(), stream())
    ft.ft_expert_combine(s.desc, 520, y.data_ptr(), s.row_of.data_ptr(), 0, back.data_ptr(), stream())
    torch.cuda.synchronize()
    assert torch.equal(y[s.row_of.long(), :100], x[:, :100]) and torch.equal(back, x)
