"""The decoder block example at lengths and budgets other than its own: tables hold what its sequences grow to, and a step beyond a table is refused on the host."""
import sys

import pytest
import torch

from test_gpu_block_example import PATH, load


def test_a_step_beyond_the_table_is_refused():
    ex = load()
    b = ex.Block.__new__(ex.Block)
    b.score = torch.zeros((1, 2, 64))
    lens = torch.tensor([64], dtype=torch.int32)
    with pytest.raises(ValueError, match="65 tokens"):
        b.decode(None, None, None, None, lens, 65, lens, None, None)


@pytest.mark.parametrize("args", [["--steps", "0"], ["--budget", "0"], ["--budget", "-3"]])
def test_no_steps_and_no_budget_are_refused(monkeypatch, capsys, args):
    monkeypatch.setattr(sys, "argv", [PATH, *args])
    with pytest.raises(SystemExit):
        load().main()
    assert "1 or more" in capsys.readouterr().err


@pytest.mark.gpu
@pytest.mark.parametrize("steps,budget", [(70, 64), (66, 100), (5, 1), (1, 16), (64, 64)])
def test_other_lengths_and_budgets(monkeypatch, capsys, steps, budget):
    monkeypatch.setattr(sys, "argv", [PATH, "--steps", str(steps), "--budget", str(budget)])
    load().main()
    said = capsys.readouterr().out
    assert f"{[min(steps, budget)] * 3} kept of {[steps] * 3}" in said and "nan" not in said
