"""What the node sweep's command makes of the ranks' results, without a GPU: loads and qualification are stand-ins."""
import math

import torch

from paper_2605_17879_b200 import sweep_run


def passes(rows, nodes, per):
    """In place of guard.sweep_qualify: a GPU fails where its first metric's median is below 50."""
    med = rows.median(1).values
    ok = med[:, 0] >= 50
    assert nodes * per == len(rows) and rows.isfinite().all()
    return {"gpu_med": med, "fail_mask": (~ok).int(), "gpu_pass": ok.byte()}


def results(gpus, reps=3):
    return torch.full((gpus, reps, 4), 100.0), torch.arange(float(reps)).repeat(gpus, 1)


def test_agreement_takes_whole_rows_and_a_strict_majority():
    a, b, c = [1.0, 2.0], [1.0, 3.0], [0.5, 2.0]
    t = lambda *rows: torch.tensor(rows)    # noqa: E731
    assert sweep_run.agreement(t(a)) == [True]
    assert sweep_run.agreement(t(a, a)) == [True, True]
    assert sweep_run.agreement(t(a, b)) == [None, None]
    assert sweep_run.agreement(t(a, b, a)) == [True, False, True]
    assert sweep_run.agreement(t(a, b, c)) == [None] * 3          # (elementwise, [1, 2] would be the commonest)
    assert sweep_run.agreement(t(a, a, b, b)) == [None] * 4
    nan = [math.nan, 1.0]
    assert sweep_run.agreement(t(nan, nan, a)) == [True, True, False]      # bit for bit
    assert sweep_run.agreement(t([0.0], [-0.0], [0.0])) == [True, False, True]
    assert sweep_run.agreement(torch.empty(0, 3)) == []


def test_verdict():
    rows, losses = results(4)
    got = sweep_run.verdict(rows, losses, 2, 2, passes)
    assert got["gpu_pass"] == [1] * 4 and got["node_pass"] == [1, 1] and got["same_results"] == [True] * 4 and got["last_loss"] == 2.0
    assert got["medians"][3] == dict.fromkeys(sweep_run.METRICS, 100.0)
    slow = rows.clone()
    slow[1] = 10
    got = sweep_run.verdict(slow, losses, 2, 2, passes)
    assert got["gpu_pass"] == [1, 0, 1, 1] and got["node_pass"] == [0, 1] and got["fail_mask"] == [0, 1, 0, 0]
    wrong = losses.clone()
    wrong[2, 0] += 1                                               # fast, but wrong
    got = sweep_run.verdict(rows, wrong, 2, 2, passes)
    assert got["gpu_pass"] == [1, 1, 0, 1] and got["node_pass"] == [1, 0] and got["same_results"] == [True, True, False, True]
