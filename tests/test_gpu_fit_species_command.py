"""The command of the fit, as a user starts it."""
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steps", [0, 1, 20])
def test_any_number_of_steps(steps, monkeypatch, capsys):
    from paper_2506_02023_amd import fit_species as fs
    monkeypatch.setattr(sys, "argv", ["fit_species", "--structures", "4", "--cells", "3", "--steps", str(steps)])
    fs.main()
    said = capsys.readouterr().out
    assert "4 structures" in said and f"{steps} steps" in said and "largest error of the" in said
    assert ("error per atom" in said) == (steps > 0)
