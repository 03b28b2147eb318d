"""The node sweep's command on one GPU, from its arguments to its line of JSON."""
import json

import pytest

pytestmark = pytest.mark.gpu


def test_main_reports_one_gpu(capsys):
    from paper_2605_17879_b200 import sweep_run
    assert sweep_run.main(["--reps", "4", "--rows", "300", "--width", "64", "--vocab", "500"]) == 0
    got = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert got["gpus"] == 1 and got["reps"] == 4 and got["gpu_pass"] == [1] and got["node_pass"] == [1] and got["same_results"] == [True]
    assert got["load_failed"] == [False] and all(x > 0 for x in got["medians"][0].values()) and got["last_loss"] > 0


def test_main_reports_a_load_that_fails(capsys, monkeypatch):
    from paper_2605_17879_b200 import guard, sweep_run

    def runs_out(self, reps):
        raise guard.GuardError(-5, "a bounded wait ran out")
    monkeypatch.setattr(sweep_run.SweepStep, "measure", runs_out)
    assert sweep_run.main(["--reps", "4", "--rows", "300", "--width", "64", "--vocab", "500"]) == 1
    printed = capsys.readouterr()
    got = json.loads(printed.out.strip().splitlines()[-1])
    assert got["gpu_pass"] == [0] and got["load_failed"] == [True] and "ran out" in printed.err
