"""Options of a plan do not go with a product that has none."""
import sys

import pytest


@pytest.mark.parametrize("option", [["--baseline"], ["--force", "256,256,128,128"], ["--zeta", "2"], ["--copy-mb", "1"]])
def test_options_of_a_plan_are_refused(monkeypatch, capsys, option):
    import run_shape
    monkeypatch.setattr(sys, "argv", ["run_shape.py", "--m", "16", "--n", "16", "--k", "16", "--dtype", "i8"] + option)
    with pytest.raises(SystemExit) as e:
        run_shape.main()
    assert e.value.code == 2 and "--dtype i8 has no plan" in capsys.readouterr().err
