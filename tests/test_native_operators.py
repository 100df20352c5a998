"""The native calls of 8-bit products and of tokens sorted by expert against the ctypes functions that they stand in for (what they call for
keywords): the same errors, for arguments that they read themselves and for those that they hand on.  No call reaches a GPU."""
import ctypes as C

import pytest

import paper_2407_21418_amd as ft
from paper_2407_21418_amd import binding

P = 1 << 20
CALLS = {
    "ft_i8_quantize": (ft.ft_quant_desc(cols=16), 0, P, P, P, 0),
    "ft_i8_matmul": (ft.ft_i8_desc(n=16, k=16), 0, P, P, P, P, 0, P, 0),
    "ft_i8_matmul_experts": (ft.ft_i8_desc(n=16, k=16, experts=2), 0, P, P, P, 0, 1, P, P, 0, P, 0),
    "ft_expert_sort": (ft.ft_expert_desc(experts=2, top_k=0), 4, P, P, P, P, 0, 0, 0),
    "ft_expert_gather": (ft.ft_expert_desc(experts=2, top_k=1, cols=8), 0, P, P, P, 0),
    "ft_expert_combine": (ft.ft_expert_desc(experts=2, top_k=1, cols=8), 0, P, P, P, P, 0),
    "ft_expert_combine_grad": (ft.ft_expert_desc(experts=2, top_k=1, cols=8), 0, P, P, P, P, P, P, 0),
}


def outcome(f, *a, **kw):
    try:
        return ("value", f(*a, **kw))
    except Exception as e:
        return (type(e), getattr(e, "status", None))


def test_the_built_calls_are_in_use():
    assert set(CALLS) == set(binding._NATIVE_OPS)
    for name in CALLS:
        assert type(getattr(ft, name)).__name__ == "builtin_function_or_method"


@pytest.mark.parametrize("name", CALLS)
def test_same_outcomes(name):
    f, args = getattr(ft, name), CALLS[name]
    want = ("value", None) if name != "ft_expert_sort" else (ft.FtError, ft.FT_ERR_INVALID_ARG)
    assert outcome(f, *args) == outcome(f, *args[:-1]) == outcome(f, *args[:-1], stream=0) == want
    odd = type(args[0])(struct_size=4)
    tries = [(odd,) + args[1:], (None,) + args[1:], (3,) + args[1:], (ft.ft_shape(m=1),) + args[1:], args[:-2], args + (0,)]
    for i in range(1, len(args)):
        tries += [args[:i] + (v,) + args[i + 1:] for v in (None, 1, -1, 2 ** 31, 2 ** 64 + 16, 16.0, "x", True, C.c_void_p(16), 0) if not (i == 1 and v not in (None, 0, 16.0, "x", 2 ** 31))]
    for a in tries:
        native = outcome(f, *a)
        ctypes_ = outcome(f, *a[:-1], stream=a[-1]) if len(a) == len(args) else native
        assert native == ctypes_, a[1:]


@pytest.mark.parametrize("name", CALLS)
def test_refusals_have_the_call_s_name(name):
    args = CALLS[name]
    with pytest.raises(ft.FtError, match=name + ":"):
        getattr(ft, name)(type(args[0])(struct_size=4), *args[1:])
