"""The calls of the framework in perf/operators.py against the operators' definitions in 64 bits: no precision is lost on the way from one call to the next.

The plain form rounds its result to the type once.  The calls round the rows of the second product and their weighted sum: two roundings of the same kind, the
first spread over a token's rows, so that a result is at most twice as far from 64 bits in the 2-norm as the plain form's, and 1.4 times where the two are independent.  A
32-bit output has its sums in another order: within 2^-20 of its norm.  Gates and values that are rounded to 16 bits before they are quantised are
six times as far off and more."""
import importlib.util
import os
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def operators():
    spec = importlib.util.spec_from_file_location("operators_under_test", os.path.join(ROOT, "perf", "operators.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def outputs(operators, case, seed, own):
    operators.own = own
    try:
        got = operators.run(operators.prepare(case, seed))
        torch.cuda.synchronize()
        return {k: v.clone() for k, v in got.items()}
    finally:
        operators.own = False


def check(operators, case, seed):
    own, plain, exact = outputs(operators, case, seed, True), outputs(operators, case, seed, False), operators.exact(case, seed)
    assert set(own) == set(plain)
    for name, want in exact.items():
        if not want.dtype.is_floating_point:
            assert torch.equal(own[name], plain[name]) and torch.equal(own[name].long(), want.long()), name
            continue
        want = want.double()
        off = [float((got[name].double() - want).norm() / want.norm()) for got in (own, plain)] if want.numel() and bool(want.any()) else [float(own[name].double().abs().sum()), 0.0]
        assert off[0] <= 2 * off[1] + 2.0 ** -20, (name, off)


@pytest.mark.parametrize("name", ["linear 1x4096x4096", "linear 77x768x768", "linear 403x1003x1001", "permute 5 top 2", "permute 1234 top 6 grad", "experts 4 top 2", "experts 64 top 4",
                                  "experts 1000 top 2 odd"])
def test_listed(operators, name):
    check(operators, next(c for c in operators.listed() if c["name"] == name), 7)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,top_k,experts,cols,ffn,padded", [(1, 1, 4, 64, 64, 0), (37, 3, 9, 517, 130, 5), (600, 8, 32, 512, 704, 0)])
def test_layers(operators, dtype, tokens, top_k, experts, cols, ffn, padded):
    check(operators, dict(kind="experts", tokens=tokens, top_k=top_k, experts=experts, cols=cols, ffn=ffn, dtype=dtype, padded=padded), 9)


def test_drawn(operators):
    rng, done = random.Random(5), 0
    while done < 6:
        case = operators.draw(rng)
        w = operators.work(case)
        if w["bytes"] > 2e8 or w["flops"] > 2e11:
            continue
        check(operators, case, done)
        done += 1
