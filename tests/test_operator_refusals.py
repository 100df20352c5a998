"""Matmuls in 8-bit integers and tokens sorted by expert: what their entry points turn down, and calls with nothing to do.  None of these
calls reaches a GPU."""
import pytest

import paper_2407_21418_amd as ft

BAD, NOT_HERE = ft.FT_ERR_INVALID_ARG, ft.FT_ERR_UNSUPPORTED
P = 1 << 20                               # addresses that nobody reads
QUANT = dict(cols=100)
PRODUCT = dict(n=64, k=100)
GROUPED = dict(n=64, k=100, experts=4)
MOVE = dict(experts=4, top_k=2, cols=64)


def status(f, *args):
    try:
        f(*args)
    except ft.FtError as e:
        return e.status
    return ft.FT_OK


def quantize(desc=None, rows=3, X=P, Q=P, scale=P, **more):
    return status(ft.ft_i8_quantize, desc or ft.ft_quant_desc(**{**QUANT, **more}), rows, X, Q, scale)


@pytest.mark.parametrize("more,want", [
    (dict(cols=0), BAD), (dict(cols=(1 << 20) + 1), NOT_HERE), (dict(dtype=3), BAD), (dict(act=2), BAD), (dict(struct_size=4), BAD), (dict(ldx=99), BAD),
    (dict(ldx=199, act=ft.FT_ACT_SILU_MUL), BAD), (dict(ldq=96), BAD), (dict(ldq=120), BAD), (dict(ldx=1 << 23), NOT_HERE), (dict(ldq=1 << 23), NOT_HERE),
    (dict(rows=1 << 31), NOT_HERE), (dict(X=0), BAD), (dict(Q=0), BAD), (dict(scale=0), BAD), (dict(X=P + 1), BAD), (dict(Q=P + 8), BAD), (dict(scale=P + 2), BAD), (dict(X=P + 2, dtype=ft.FT_F32), BAD)])
def test_quantize(more, want):
    assert quantize(**more) == want


def test_quantize_without_rows():
    assert quantize(rows=0) == quantize(rows=0, X=0, Q=0, scale=0) == ft.FT_OK
    assert quantize(rows=0, cols=0) == BAD


def matmul(m=5, A=P, sa=P, B=P, sb=P, bias=0, C=P, **more):
    return status(ft.ft_i8_matmul, ft.ft_i8_desc(**{**PRODUCT, **more}), m, A, sa, B, sb, bias, C)


def grouped(rows=5, offsets=P, A=P, sa=P, a_row=0, a_rows=5, B=P, sb=P, bias=0, C=P, **more):
    return status(ft.ft_i8_matmul_experts, ft.ft_i8_desc(**{**GROUPED, **more}), rows, offsets, A, sa, a_row, a_rows, B, sb, bias, C)


PRODUCT_REFUSALS = [
    (dict(n=0), BAD), (dict(k=0), BAD), (dict(n=1 << 20), NOT_HERE), (dict(k=131072), NOT_HERE), (dict(dtype=ft.FT_F32), BAD), (dict(out_dtype=2), BAD), (dict(epilogue=3), BAD), (dict(n=63, epilogue=ft.FT_EPI_SILU_MUL), BAD), (dict(epilogue=ft.FT_EPI_SILU_MUL, bias=P), BAD), (dict(epilogue=ft.FT_EPI_SILU_MUL, ldc=31), BAD),
    (dict(struct_size=4), BAD), (dict(lda=96), BAD), (dict(ldb=96), BAD), (dict(ldc=63), BAD), (dict(lda=120), BAD), (dict(ldb=104), BAD), (dict(lda=(1 << 20) + 16), NOT_HERE),
    (dict(ldb=(1 << 20) + 16), NOT_HERE), (dict(ldc=(1 << 22) + 1), NOT_HERE), (dict(bias=P), BAD), (dict(epilogue=ft.FT_EPI_BIAS), BAD), (dict(A=0), BAD), (dict(B=0), BAD), (dict(C=0), BAD),
    (dict(sa=0), BAD), (dict(sb=0), BAD), (dict(A=P + 8), BAD), (dict(B=P + 4), BAD), (dict(C=P + 2), BAD), (dict(C=P + 1, out_dtype=ft.FT_OUT_SAME), BAD), (dict(sa=P + 1), BAD), (dict(sb=P + 2), BAD),
    (dict(epilogue=ft.FT_EPI_BIAS, bias=P + 2), BAD)]


@pytest.mark.parametrize("more,want", PRODUCT_REFUSALS + [(dict(experts=1), BAD), (dict(m=1 << 31), NOT_HERE)])
def test_matmul(more, want):
    assert matmul(**more) == want


@pytest.mark.parametrize("more,want", PRODUCT_REFUSALS + [
    (dict(experts=0), BAD), (dict(experts=1025), NOT_HERE), (dict(rows=1 << 31), NOT_HERE), (dict(offsets=0), BAD), (dict(offsets=P + 2), BAD), (dict(a_row=P + 1), BAD), (dict(a_rows=0), BAD),
    (dict(a_rows=1 << 25), NOT_HERE)])
def test_matmul_experts(more, want):
    assert grouped(**more) == want


def test_products_without_rows():
    assert matmul(m=0) == matmul(m=0, A=0, B=0, C=0, sa=0, sb=0) == grouped(rows=0) == grouped(rows=0, offsets=0, A=0, C=0, a_rows=0) == ft.FT_OK
    assert matmul(m=0, n=0) == matmul(m=0, bias=P) == BAD


def workspace(tokens, **more):
    return ft.ft_expert_workspace(ft.ft_expert_desc(**{**MOVE, **more}), tokens)


def sort(tokens=5, ids=P, offsets=P, row_token=P, row_of=P, ws=P, ws_bytes=1 << 30, **more):
    return status(ft.ft_expert_sort, ft.ft_expert_desc(**{**MOVE, **more}), tokens, ids, offsets, row_token, row_of, ws, ws_bytes)


SHAPE_REFUSALS = [(dict(experts=0), BAD), (dict(top_k=0), BAD), (dict(experts=1025), NOT_HERE), (dict(top_k=33), NOT_HERE), (dict(struct_size=4), BAD), (dict(tokens=1 << 30), NOT_HERE)]


@pytest.mark.parametrize("more,want", SHAPE_REFUSALS + [
    (dict(ids=0), BAD), (dict(offsets=0), BAD), (dict(row_token=0), BAD), (dict(row_of=0), BAD), (dict(ids=P + 1), BAD), (dict(offsets=P + 2), BAD), (dict(row_token=P + 1), BAD), (dict(row_of=P + 3), BAD),
    (dict(tokens=1 << 20, ws=0), BAD), (dict(tokens=1 << 20, ws=P + 4), BAD), (dict(tokens=1 << 20, ws_bytes=4095), BAD), (dict(tokens=0, offsets=0), BAD)])
def test_sort(more, want):
    assert sort(**more) == want


def test_workspace():
    assert workspace(0) == workspace(5) == workspace(4096) == 0
    assert 0 < workspace(100000) <= workspace(1 << 20) <= workspace((1 << 30) - 1) <= 4096
    for more, want in SHAPE_REFUSALS:
        more = dict(more)
        assert status(lambda: workspace(more.pop("tokens", 5), **more)) == want


def gather(tokens=5, X=P, row_of=P, Y=P, **more):
    return status(ft.ft_expert_gather, ft.ft_expert_desc(**{**MOVE, **more}), tokens, X, row_of, Y)


def combine(tokens=5, X=P, row_of=P, Y=P, w=P, **more):
    return status(ft.ft_expert_combine, ft.ft_expert_desc(**{**MOVE, **more}), tokens, Y, row_of, w, X)


def grad(tokens=5, X=P, row_of=P, Y=P, w=P, dY=P, dw=P, **more):
    return status(ft.ft_expert_combine_grad, ft.ft_expert_desc(**{**MOVE, **more}), tokens, X, Y, row_of, w, dY, dw)


@pytest.mark.parametrize("call", [gather, combine, grad])
@pytest.mark.parametrize("more,want", SHAPE_REFUSALS + [
    (dict(cols=0), BAD), (dict(cols=(1 << 20) + 1), NOT_HERE), (dict(dtype=3), BAD), (dict(ld_token=63), BAD), (dict(ld_row=63), BAD), (dict(ld_token=1 << 23), NOT_HERE), (dict(ld_row=1 << 23), NOT_HERE),
    (dict(X=0), BAD), (dict(Y=0), BAD), (dict(row_of=0), BAD), (dict(X=P + 1), BAD), (dict(Y=P + 1), BAD), (dict(row_of=P + 2), BAD), (dict(X=P + 2, dtype=ft.FT_F32), BAD),
    (dict(Y=P + 2, dtype=ft.FT_F32), BAD)])
def test_moves(call, more, want):
    assert call(**more) == want


def test_gradient_and_weights():
    assert combine(w=P + 2) == grad(w=P + 1) == grad(dw=P + 2) == grad(dY=0) == grad(dY=P + 1) == BAD
    assert gather(tokens=0, X=0, Y=0, row_of=0) == combine(tokens=0, X=0, Y=0, row_of=0) == grad(tokens=0, X=0, Y=0, row_of=0, dY=0) == ft.FT_OK
