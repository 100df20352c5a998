"""The measurement commands' 8-bit workloads run, and say what they measured."""
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_one_shape_in_8_bits(monkeypatch, capsys):
    import run_shape
    monkeypatch.setattr(sys, "argv", ["run_shape.py", "--m", "77", "--n", "200", "--k", "100", "--dtype", "i8", "--iters", "3", "--ring-mb", "0.1"])
    run_shape.main()
    assert capsys.readouterr().out.startswith("77x200x100 i8: quantise ")


@pytest.mark.parametrize("tokens,top_k,experts", [(1, 2, 4), (50, 3, 9)])
def test_a_ragged_batch_of_experts(tokens, top_k, experts):
    import run_ragged
    rows = run_ragged.measure_experts(experts=experts, tokens=tokens, top_k=top_k, cols=96, inner=40, iters=2, draws=2)
    assert [r["draw"] for r in rows] == [0, 1]
    for r in rows:
        assert min(r["us_layer"], r["us_grouped"], r["us_padded"], r["us_looped"]) > 0
        assert r["most_rows"] * experts >= tokens * top_k and r["padded_work_ratio"] >= 1
