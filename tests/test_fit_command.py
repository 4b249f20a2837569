"""Refusals of the fitting example's command, which come before a GPU is needed."""
import pytest

from paper_2606_12950_amd import fit as F


@pytest.mark.parametrize("steps", ["0", "-3"])
def test_no_steps(steps, capsys):
    with pytest.raises(SystemExit) as e:
        F.main(["--steps", steps])
    assert e.value.code == 2 and "--steps" in capsys.readouterr().err
