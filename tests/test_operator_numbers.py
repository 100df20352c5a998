"""Numbers of rows, tokens and bytes beyond the library's types: refused, where ctypes would drop the bits that its type lacks (2^32 rows were none, and -1 bytes of workspace
enough of them).  No call reaches a GPU."""
import pytest

import paper_2407_21418_amd as ft

P = 1 << 20
CALLS = {                                                    # f(number, more of them by keyword)
    "ft_i8_quantize": lambda n, **kw: ft.ft_i8_quantize(ft.ft_quant_desc(cols=16), n, P, P, P, **kw),
    "ft_i8_matmul": lambda n, **kw: ft.ft_i8_matmul(ft.ft_i8_desc(n=16, k=16), n, P, P, P, P, 0, P, **kw),
    "ft_i8_matmul_experts": lambda n, **kw: ft.ft_i8_matmul_experts(ft.ft_i8_desc(n=16, k=16, experts=2), n, P, P, P, 0, 1, P, P, 0, P, **kw),
    "rows of A": lambda n, **kw: ft.ft_i8_matmul_experts(ft.ft_i8_desc(n=16, k=16, experts=2), 0, P, P, P, 0, n, P, P, 0, P, **kw),
    "ft_expert_sort": lambda n, **kw: ft.ft_expert_sort(ft.ft_expert_desc(experts=2, top_k=1), n, P, P, P, P, P, 1 << 20, **kw),
    "ft_expert_gather": lambda n, **kw: ft.ft_expert_gather(ft.ft_expert_desc(experts=2, top_k=1, cols=8), n, P, P, P, **kw),
    "ft_expert_combine": lambda n, **kw: ft.ft_expert_combine(ft.ft_expert_desc(experts=2, top_k=1, cols=8), n, P, P, 0, P, **kw),
    "ft_expert_combine_grad": lambda n, **kw: ft.ft_expert_combine_grad(ft.ft_expert_desc(experts=2, top_k=1, cols=8), n, P, P, P, 0, P, 0, **kw),
}


def status(f, *a, **kw):
    try:
        f(*a, **kw)
    except ft.FtError as e:
        return e.status
    return ft.FT_OK


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("by_keyword", [False, True])
def test_counts(name, by_keyword):
    """By keyword the ctypes functions are called, else the native ones."""
    kw = dict(stream=0) if by_keyword else {}
    for n in (1 << 32, (1 << 32) + 5, 1 << 64, (1 << 64) + 16, 1 << 70):
        assert status(CALLS[name], n, **kw) == ft.FT_ERR_UNSUPPORTED, n
    for n in (-1, -(1 << 32), 5 - (1 << 32), -(1 << 64), -(1 << 70)):
        assert status(CALLS[name], n, **kw) == ft.FT_ERR_INVALID_ARG, n


@pytest.mark.parametrize("by_keyword", [False, True])
def test_bytes_of_workspace(by_keyword):
    kw = dict(stream=0) if by_keyword else {}
    f = lambda n: status(ft.ft_expert_sort, ft.ft_expert_desc(experts=2, top_k=1), 1 << 20, P, P, P, P, P, n, **kw)  # noqa: E731
    assert f(-1) == f(-(1 << 70)) == f(0) == f(5) == ft.FT_ERR_INVALID_ARG and f(1 << 64) == f((1 << 64) + (1 << 20)) == ft.FT_ERR_UNSUPPORTED


def test_workspace():
    f = lambda n: status(ft.ft_expert_workspace, ft.ft_expert_desc(experts=2, top_k=1), n)  # noqa: E731
    assert f(1 << 32) == f((1 << 32) + 5) == ft.FT_ERR_UNSUPPORTED and f(-1) == ft.FT_ERR_INVALID_ARG and f(1 << 20) == ft.FT_OK
